"""The workspace of attention over the 8-bit cache: what is enough for the largest sequences, max_new and max_len is enough for every batch within them (no GPU takes part)."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

from paper_2411_05007_amd import svdq as S

HERE = os.path.dirname(os.path.abspath(__file__))
WITHIN = r"""
#include <stdio.h>
#include <random>
#include "layout.h"
using namespace svdq;
int main() {
    std::mt19937 gen(1);
    auto upto = [&](double most) {      // 0 .. most, over its logarithm
        return (int)(std::exp(std::uniform_real_distribution<double>(0.0, std::log(most + 1.0))(gen)) - 0.999999);
    };
    for (int i = 0; i < 3000000; ++i) {
        const int heads = 1 + upto(40), group = 1 + upto(40), dim = 64 << gen() % 3, sequences = 1 + upto(5000), max_new = upto(70000), max_len = upto(1 << 30);
        const size_t room = kv_workspace_bytes(sequences, heads, group, dim, max_new, max_len);
        const int b = 1 + upto(sequences - 1), n = upto(max_new), l = upto(max_len), near = gen() % 2 ? max_len - upto(max_len / 8) : l;
        if (kv_workspace_bytes(b, heads, group, dim, n, near) > room) return printf("query: %d %d %d, %d %d %d of %d %d %d\n", heads, group, dim, b, n, near, sequences, max_new, max_len), 1;
        const long long tokens = gen() % 4 ? (long long)((double)b * n * (gen() % 1001) / 1000.0) : (long long)b * n + gen() % 50;
        if (plan_kv_attention(b, heads, group, dim, n, near, gen() % 3 ? 0 : 1 + upto(1 << 20), tokens).total > room)
            return printf("call: %d %d %d, %d %d %d (%lld) of %d %d %d\n", heads, group, dim, b, n, near, tokens, sequences, max_new, max_len), 1;
    }
    return printf("ok\n"), 0;
}
"""


def test_a_batch_within_another_needs_no_more(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "within.cpp", tmp_path / "within"
    src.write_text("#include <cmath>\n" + WITHIN)
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", os.path.join(os.path.dirname(HERE), "paper_2411_05007_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


def test_the_entry_point_s_size_grows_with_its_arguments():
    if not os.path.exists(S.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    size = lambda heads, q_heads, dim, *a: S.lib().svdq_kv_attention_workspace_bytes(C.byref(S.KVShape(heads, dim, 64)), q_heads, *a)
    assert size(8, 32, 128, 1, 1, 8180) <= size(8, 32, 128, 1, 1, 8277)
    assert size(8, 32, 128, 2, 1, 4000) <= size(8, 32, 128, 3, 1, 4000)
    rng = random.Random(2)
    for _ in range(300):
        heads, group, dim = rng.choice([1, 2, 8, 24]), rng.choice([1, 2, 4, 8, 17]), rng.choice([64, 128, 256])
        at = [rng.choice([1, 2, 40]), rng.choice([1, 2, 5, 60, 300]), rng.choice([1, 900, 5000])]
        last = 0
        for _ in range(60):
            i = rng.randrange(3)
            at[i] += rng.choice([1, 7, at[i] // 3 + 1])
            now = size(heads, heads * group, dim, *[min(x, 1 << 29) for x in at])
            assert now >= last and now > 0, (heads, group, dim, at)
            last = now


def test_sizes_stay_near_what_a_call_uses():
    """A guard against a bound that is only large: single tokens take the sums of one part for each 4096 keys, sequence and key head, or of 256 parts; chunks 34 MB and the same of sixteen rows."""
    size = lambda *a: S.lib().svdq_kv_attention_workspace_bytes(C.byref(S.KVShape(8, 128, 64)), 32, *a)
    assert size(64, 1, 1000) == 256 and size(64, 1, 1024) == 256
    assert size(1, 1, 4000) <= 256 * (4 * 130 * 4 + 8) + 512
    assert size(64, 1, 16384) <= 64 * 8 * 4 * (4 * 130 * 4 + 8) + 512
    assert size(1, 8192, 16384) <= 34 * 2 ** 20
    assert size(6, 2111, 3611) <= 34 * 2 ** 20 + 256 * (16 * 130 * 4 + 8) + 1024
