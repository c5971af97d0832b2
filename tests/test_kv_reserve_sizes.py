"""The workspace of a reservation at the largest pools and tables: 64-bit sizes, by the entry point's answers (no GPU is needed)."""
import os

import pytest

from paper_2411_05007_amd import svdq as S


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return S.lib()


@pytest.mark.parametrize("pages", [1, 1024, 1025, 2 ** 30, 2 ** 31 - 1024, 2 ** 31 - 1023, 2 ** 31 - 1])
@pytest.mark.parametrize("sequences,width", [(0, 0), (3, 2), (65535, 64), (3, 2 ** 31 - 64), (3, 2 ** 31 - 63), (3, 2 ** 31 - 1)])
def test_the_workspace_grows_with_the_pool_and_the_table(lib, pages, sequences, width):
    got = lib.svdq_kv_pages_reserve_workspace_bytes(S.KVPoolDev(1 << 28, pages, 64), sequences, width)
    # a bit a page and a count for each 1024 of them; two numbers a sequence and a bit an entry; five parts that begin at multiples of 256
    slices = -(-pages // 1024)
    least = slices * (128 + 4) + sequences * (8 + 8 * -(-width // 64))
    assert least <= got <= least + 5 * 255
