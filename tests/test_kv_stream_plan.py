"""How attention with norms or first tokens that stay visible is cut (csrc/layout.h, plan_kv_attention with `wide`): the bounds of tests/test_kv_plan.py, and which kernels it takes."""
import os
import shutil
import subprocess

import pytest

from tests import test_kv_plan as P

CALL = "max_new, max_len, window, tokens), asked"


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    assert CALL in P.BOUNDS and "a[6], a[7]);" in P.BOUNDS
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "bounds.cpp", d / "bounds"
    src.write_text(P.BOUNDS.replace(CALL, CALL.replace("tokens)", "tokens, true)")).replace("a[6], a[7]);", "a[6], a[7], true);"))
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(os.path.dirname(P.HERE), "paper_2411_05007_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return lambda *a: subprocess.run([str(exe), *map(str, a)], capture_output=True, text=True)


def test_plans_stay_within_the_workspace_and_the_kernels_bounds(plan):
    r = plan()
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


@pytest.mark.parametrize("sequences,heads,group,dim,max_new,max_len,window,tokens,want", [
    (1, 8, 4, 128, 8192, 24576, 8192, 8192, "256 1"), (1, 8, 4, 128, 8192, 24576, 2048, 8192, "256 1"), (1, 8, 4, 128, 8192, 24576, 2047, 8192, "128 1"),
    (8, 8, 2, 128, 4096, 8192, 2048, 32768, "128 1"), (1, 24, 1, 128, 4608, 12608, 8192, 4608, "256 1"), (1, 8, 4, 128, 8192, 24576, 0, 8192, "256 1"),
    (1, 8, 4, 64, 8192, 24576, 8192, 8192, "128 1"), (2, 8, 4, 128, 8192, 24576, 8192, 8193, "128 1"), (64, 8, 4, 128, 1, 32768, 8256, 64, "few 2"),
])
def test_the_kernels_in_a_window(plan, sequences, heads, group, dim, max_new, max_len, window, tokens, want):
    assert plan(sequences, heads, group, dim, max_new, max_len, window, tokens).stdout.strip().split(", ")[0] == want
