"""What the entry points for streams and branches on the paged 8-bit cache refuse, by their return values: nothing is launched and no pointer is followed, so no GPU is needed."""
import ctypes as C
import os

import pytest

from paper_2411_05007_amd import svdq as S

AT = 0x10000000
EINVAL, EUNSUPPORTED, ENOSPACE = -1, -2, -4
CACHE = S.KVCacheDev(AT, AT, AT, AT, 4, S.KVShape(2, 128, 64))
BATCH = S.KVBatchDev(AT, AT, AT, 3, 2, 5, 4, 100)
NONE = S.KVBatchDev(AT, AT, AT, 0, 2, 0, 0, 0)
ROWS = S.KVRowsDev(AT, 256, 128)
FINE = (AT, AT, AT, AT, 3, 1, 1e-6)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return S.lib()


def norm(i=None, value=None):
    f = list(FINE)
    if i is not None:
        f[i] = value
    return S.KVNormDev(*f)


@pytest.mark.parametrize("i,value", [(0, AT + 4), (1, AT + 8), (2, AT + 1), (3, AT + 12), (4, -1), (6, 0.0), (6, -1e-6), (6, 1e-31), (6, float("inf")), (6, float("nan"))])
def test_norms_that_are_refused(lib, i, value):
    for batch in (BATCH, NONE):      # (also where there is nothing to do)
        assert lib.svdq_kv_append_normed(CACHE, batch, norm(i, value), None, ROWS, ROWS, None) == EINVAL
        assert lib.svdq_kv_attention_normed(CACHE, batch, norm(i, value), None, ROWS, 4, 0.1, 1, 7, 3, AT, AT, C.c_size_t(1 << 40), None) == EINVAL


def test_norms_that_are_taken(lib):
    for n in (norm(), norm(0, None), norm(1, None), norm(2, None), norm(3, None), norm(4, 0), norm(5, 0), norm(6, 1e-30), norm(6, 3e38), None):
        assert lib.svdq_kv_append_normed(CACHE, NONE, n, None, ROWS, ROWS, None) == 0
        assert lib.svdq_kv_attention_normed(CACHE, NONE, n, None, ROWS, 4, 0.1, 1, 7, 3, AT, AT, C.c_size_t(1 << 40), None) == 0


def test_first_tokens_below_zero_are_refused(lib):
    call = lambda window, sinks, size=1 << 40: lib.svdq_kv_attention_normed(CACHE, BATCH, None, None, ROWS, 4, 0.1, 1, window, sinks, AT, AT, C.c_size_t(size), None)
    assert call(7, -1) == EINVAL and call(-1, 7) == EINVAL and call(0, -1) == EINVAL
    need = lib.svdq_kv_attention_workspace_bytes(CACHE.shape, 4, 3, 4, 100)
    for sinks in (0, 3, 2 ** 31 - 1):
        assert call(7, sinks, need - 1) == ENOSPACE


def test_the_plain_entry_points_refuse_as_before(lib):
    assert lib.svdq_kv_append(CACHE, BATCH, None, S.KVRowsDev(AT + 2, 256, 128), ROWS, None) == EINVAL
    assert lib.svdq_kv_attention(CACHE, BATCH, None, ROWS, 3, 0.1, 1, 0, AT, AT, C.c_size_t(1 << 40), None) == EINVAL
