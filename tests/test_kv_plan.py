"""How attention over the 8-bit cache is cut (csrc/layout.h, plan_kv_attention): the bounds that the kernels and the workspace rely on, and which kernels the GPU
tests reach."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2411_05007_amd import svdq as S

HERE = os.path.dirname(os.path.abspath(__file__))
BOUNDS = r"""
#include <stdio.h>
#include <stdlib.h>
#include <initializer_list>
#include "layout.h"
using namespace svdq;
static const char *wrong(const KvPlan &p, const KvPlan &asked, int sequences, int heads, int group, int dim, int max_new, int max_len, long long tokens) {
    if (p.many != asked.many || (!p.many && !p.few) || (p.few && !asked.few)) return "a window or the number of tokens changes the kernel";
    if (p.total > asked.total) return "more workspace than was asked for";
    const long long rows = p.many ? kKvFewRows : (long long)max_new * group;
    size_t at = 0;
    if (p.many) {
        if (p.tile_rows != 128 && p.tile_rows != 256) return "rows of a tile";
        if (p.tile_rows == 256 && (dim != 128 || p.parts != 1)) return "a tile of 256 rows";
        if (p.parts < 1 || p.parts > 16) return "parts";
        if (p.parts > 1) {
            const size_t all = (size_t)p.parts * tokens * heads * group;
            if (p.ml_off < all * dim * 4 || p.ml_off % 256 != 0 || p.total < p.ml_off + all * 8) return "room for the parts";
            at = p.ml_off + all * 8;
        }
    }
    if (p.few) {
        if (p.chunks < 1 || p.chunks > kKvMostChunks || p.chunk_blocks < 1) return "chunks";
        if (p.row_cap > 16 || (!p.many && (long long)p.row_tiles * 16 < rows) || (p.many && p.row_tiles != 1)) return "rows";
        if (p.row_cap < (rows < 16 ? rows : 16) && p.row_cap < (long long)max_new * group) return "rows of a tile of few";
        if (p.chunks > asked.chunks) return "more chunks than the workspace holds";
        if (p.chunks > 1) {
            const size_t parts = (size_t)sequences * p.row_tiles * heads * p.chunks;
            if (p.few_off < at || p.few_off % 256 != 0 || p.words_off < p.few_off + parts * p.row_cap * (dim + 2) * 4 || p.words_off % 256 != 0) return "place of the words";
            if (p.total < p.words_off + parts * 8) return "room for the words";
        }
    }
    return nullptr;
}
int main(int argc, char **argv) {
    if (argc > 1) {
        int a[8];
        for (int i = 0; i < 8; ++i) a[i] = atoi(argv[i + 1]);
        const KvPlan p = plan_kv_attention(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
        if (p.many) printf("%d %d%s", p.tile_rows, p.parts, p.few ? ", " : "\n");
        return p.few ? printf("few %d\n", p.chunks) : 0, 0;
    }
    for (int sequences : {1, 2, 5, 33, 64, 700, 65535})
        for (int heads : {1, 2, 8, 40})
            for (int group : {1, 4, 7, 40})
                for (int dim : {64, 128, 256})
                    for (int max_new : {0, 1, 2, 5, 16, 17, 60, 128, 129, 700, 4608, 70000})
                        for (int max_len : {0, 1, 31, 33, 500, 1025, 4096, 8192, 50001, 1 << 20, 1 << 30}) {
                            const KvPlan asked = plan_kv_attention(sequences, heads, group, dim, max_new, max_len, 0, -1);
                            const long long most = (long long)sequences * max_new;
                            for (int window : {0, 1, 64, 1000, 5000, 100000, 0x7fffffff})
                                for (long long tokens : {most, most / 2, most / 7, max_new + sequences - 1ll, 1ll, most + 5}) {
                                    const char *w = wrong(plan_kv_attention(sequences, heads, group, dim, max_new, max_len, window, tokens), asked, sequences, heads, group, dim, max_new, max_len, tokens);
                                    if (w) return printf("%s: %d sequences, %d x %d heads of %d, %d of %d, window %d, %lld tokens\n", w, sequences, heads, group, dim, max_new, max_len, window, tokens), 1;
                                }
                        }
    return printf("ok\n"), 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "bounds.cpp", d / "bounds"
    src.write_text(BOUNDS)
    subprocess.run([cxx, "-std=c++17", "-O1", "-I", os.path.join(os.path.dirname(HERE), "paper_2411_05007_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    return lambda *a: subprocess.run([str(exe), *map(str, a)], capture_output=True, text=True)


def test_plans_stay_within_the_workspace_and_the_kernels_bounds(plan):
    r = plan()
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


@pytest.mark.parametrize("sequences,heads,group,dim,max_new,max_len,window,tokens,want", [
    (64, 8, 4, 128, 1, 500, 0, 64, "few 1"), (1, 1, 4, 128, 1, 5001, 0, 1, "few 20"), (1, 1, 4, 64, 1, 2201600, 0, 1, "few 256"),
    (32, 8, 1, 128, 256, 4200, 0, 8192, "256 1"), (4, 4, 2, 128, 4100, 4100, 0, 16400, "256 1"),
    (24, 8, 2, 128, 199, 2800, 0, 3300, "128 1"), (24, 12, 1, 64, 399, 2999, 65, 7000, "128 1"), (40, 2, 4, 256, 199, 2799, 0, 5000, "128 1"),
    (2, 2, 4, 128, 300, 8000, 0, 600, "128 12"), (2, 2, 4, 128, 300, 8000, 0, 337, "128 15"), (1, 1, 8, 128, 2000, 2000, 0, 2000, "128 3"),
    (2, 3, 4, 64, 700, 12000, 0, 1350, "128 3"), (6, 2, 2, 256, 600, 3000, 0, 3600, "128 2"), (150, 4, 2, 128, 60, 659, 0, 5400, "128 1"),
    (16, 4, 2, 128, 200, 3000, 0, 3200, "128 2"), (32, 8, 4, 128, 512, 8000, 0, 554, "128 3, few 2"), (63, 12, 1, 64, 400, 3000, 0, 794, "128 5, few 1"),
    (33, 2, 2, 256, 600, 3000, 0, 647, "128 5, few 3"), (31, 8, 8, 128, 700, 9000, 3000, 730, "128 1, few 1"), (2, 8, 4, 128, 512, 100000, 0, 513, "128 3, few 25"), (4, 2, 17, 128, 300, 8000, 0, 310, "128 5"),
])
def test_the_kernels_that_the_gpu_tests_reach(plan, sequences, heads, group, dim, max_new, max_len, window, tokens, want):
    assert plan(sequences, heads, group, dim, max_new, max_len, window, tokens).stdout.strip() == want


def test_strides_that_pass_32_bits_are_refused():
    if not os.path.exists(S.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    at = 0x10000000
    cache, batch = S.KVCacheDev(at, at, at, at, 4, S.KVShape(2, 128, 64)), S.KVBatchDev(at, at, at, 3, 2, 5, 4, 100)
    for token, head, want in (((1 << 25) + 8, 128, -2), (-128, 128, -1), (256, -128, -1)):
        rows = S.KVRowsDev(at, token, head)
        assert S.lib().svdq_kv_append(cache, batch, None, rows, rows, None) == want
        assert S.lib().svdq_kv_attention(cache, batch, None, rows, 4, 0.1, 1, 0, at, at, C.c_size_t(1 << 40), None) == want
