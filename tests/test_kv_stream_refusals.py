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


# ---- compaction ------------------------------------------------------------------------------------------------------------------------------

MOVES = dict(cu_moves=AT, from_token=AT, to_first=AT, from_table=AT, to_table=AT, sequences=3, from_width=5, to_width=4, moves=70, per_head=0)


def moves(**other):
    return S.KVMovesDev(**{**MOVES, **other})


def cache(pages=4, heads=2, dim=128, page=64, k=AT):
    return S.KVCacheDev(k, AT, AT, AT, pages, S.KVShape(heads, dim, page))


@pytest.mark.parametrize("other,want", [
    (dict(cu_moves=None), EINVAL), (dict(from_token=None), EINVAL), (dict(to_first=None), EINVAL), (dict(from_table=None), EINVAL), (dict(to_table=None), EINVAL),
    (dict(from_token=AT + 2), EINVAL), (dict(to_table=AT + 1), EINVAL), (dict(from_table=AT + 3), EINVAL), (dict(from_width=0), EINVAL), (dict(to_width=0), EINVAL),
    (dict(sequences=-1), EINVAL), (dict(moves=-1), EINVAL), (dict(from_width=-1), EINVAL), (dict(sequences=65536), EUNSUPPORTED),
    (dict(from_width=(1 << 24) + 1), EUNSUPPORTED), (dict(to_width=(1 << 24) + 1), EUNSUPPORTED),
])
def test_moves_that_are_refused(lib, other, want):
    assert lib.svdq_kv_compact(CACHE, CACHE, moves(**other), None, None, 0, None) == want


def test_caches_and_workspaces_that_do_not_fit_are_refused(lib):
    call = lambda to=CACHE, source=CACHE, m=MOVES, rope=None, at=None, size=0: lib.svdq_kv_compact(to, source, moves(**m), rope, at, C.c_size_t(size), None)
    for other in (cache(heads=4), cache(dim=64), cache(pages=0), cache(k=AT + 8), cache(dim=96), cache(page=48)):
        assert call(source=other) < 0 and call(to=other) < 0
    need = lib.svdq_kv_compact_workspace_bytes(CACHE.shape, 3, 70)
    assert need >= (70 // 32 + 6) * 2 * (64 * 128 + 2)
    assert call(at=AT, size=need - 1) == ENOSPACE and call(at=AT + 128, size=need) == EINVAL
    assert call(rope=S.KVRopeDev(AT, 5, 144, 0)) == EINVAL
    for nothing in (dict(moves=0), dict(sequences=0)):
        assert call(m=nothing) == 0 and call(source=cache(page=1024), m=nothing) == 0
    assert lib.svdq_kv_compact(None, CACHE, moves(), None, None, 0, None) == EINVAL and lib.svdq_kv_compact(CACHE, CACHE, None, None, None, 0, None) == EINVAL
    assert lib.svdq_kv_compact_workspace_bytes(S.KVShape(2, 96, 64), 3, 70) == 0 and lib.svdq_kv_compact_workspace_bytes(CACHE.shape, -1, 70) == 0
    assert lib.svdq_kv_compact_workspace_bytes(CACHE.shape, 0, 0) > 0


# ---- pages -----------------------------------------------------------------------------------------------------------------------------------


def pool(refs=AT, pages=4, page=64):
    return S.KVPoolDev(refs, pages, page)


FAR = AT + (1 << 20)


@pytest.mark.parametrize("p,want", [(pool(refs=None), EINVAL), (pool(refs=AT + 2), EINVAL), (pool(pages=0), EINVAL), (pool(pages=-3), EINVAL), (pool(page=0), EINVAL),
                                    (pool(page=16), EUNSUPPORTED), (pool(page=96), EUNSUPPORTED), (pool(page=2048), EUNSUPPORTED)])
def test_pools_that_are_refused(lib, p, want):
    assert lib.svdq_kv_pages_release(p, AT, None, None, 3, 5, None) == want
    assert lib.svdq_kv_pages_fork(p, AT, AT, 3, 5, AT, FAR, FAR, 3, 5, None) == want
    assert lib.svdq_kv_pages_reserve(p, None, BATCH, None, None, AT, C.c_size_t(1 << 40), None) == want


def test_tables_that_are_refused(lib):
    release = lambda table=AT, first=None, end=None, n=3, width=5: lib.svdq_kv_pages_release(pool(), table, first, end, n, width, None)
    assert release(table=None) == release(table=AT + 2) == release(first=AT + 1) == release(end=AT + 3) == release(n=-1) == release(width=0) == release(width=-1) == EINVAL
    assert release(n=65536) == release(width=(1 << 24) + 1) == EUNSUPPORTED
    assert release(n=0) == 0 and release(table=None, n=0) == 0
    fork = lambda f=AT, fl=AT, n=3, fw=5, parent=AT, t=FAR, tl=FAR, m=4, tw=6: lib.svdq_kv_pages_fork(pool(), f, fl, n, fw, parent, t, tl, m, tw, None)
    assert fork(f=None) == fork(fl=None) == fork(parent=None) == fork(t=None) == fork(tl=None) == fork(f=AT + 1) == fork(fl=AT + 2) == fork(tl=FAR + 2) == fork(n=-1) == EINVAL
    assert fork(t=AT) == fork(t=AT + 56) == fork(f=FAR + 92) == fork(tl=AT) == fork(tl=AT + 8) == EINVAL      # the tables, or the lengths, overlap
    assert fork(m=65536) == fork(n=65536) == fork(tw=(1 << 24) + 1) == EUNSUPPORTED
    assert fork(m=0) == 0


def test_parents_that_are_written_are_refused(lib):
    fork = lambda parent, t=FAR, tl=FAR + 4096, m=4, tw=6: lib.svdq_kv_pages_fork(pool(), AT, AT, 3, 5, parent, t, tl, m, tw, None)
    assert fork(FAR + 4096) == fork(FAR + 4096 + 12) == fork(FAR + 4096 - 12) == EINVAL      # parent and to_len: each workgroup reads the one, the first writes the other
    assert fork(FAR) == fork(FAR + 92) == fork(FAR - 12) == EINVAL                           # parent and to_table


def test_reservations_that_are_refused(lib):
    p = pool()
    need = lib.svdq_kv_pages_reserve_workspace_bytes(p, 3, 2)
    call = lambda c=CACHE, b=BATCH, copies=None, missing=None, at=AT, size=1 << 40: lib.svdq_kv_pages_reserve(p, c, b, copies, missing, at, C.c_size_t(size), None)
    batch = lambda **o: S.KVBatchDev(*{**dict(cu=AT, len=AT, table=AT, sequences=3, width=2, new=5, max_new=4, max_len=100), **o}.values())
    assert call(copies=AT + 2) == call(missing=AT + 1) == call(at=None) == call(at=AT + 128) == EINVAL
    assert call(c=cache(pages=3)) == call(c=cache(page=128)) == EINVAL
    assert call(size=need - 1) == ENOSPACE
    assert call(b=batch(cu=None)) == call(b=batch(len=None)) == call(b=batch(table=None)) == call(b=batch(sequences=-1)) == call(b=batch(new=-1)) == call(b=batch(width=0)) == EINVAL
    assert call(b=batch(table=None, new=0)) == call(b=batch(cu=None, new=0)) == EINVAL      # (no tokens: missing is counted all the same)
    assert call(b=batch(sequences=65536)) == EUNSUPPORTED
    assert call(b=batch(sequences=0), at=None, size=0) == 0
    assert lib.svdq_kv_pages_reserve_workspace_bytes(pool(pages=0), 3, 2) == 0 and lib.svdq_kv_pages_reserve_workspace_bytes(p, -1, 2) == 0
    assert lib.svdq_kv_copy_pages(CACHE, CACHE, None, 3, None) == lib.svdq_kv_copy_pages(CACHE, CACHE, AT + 1, 3, None) == lib.svdq_kv_copy_pages(CACHE, CACHE, AT, -1, None) == EINVAL
    for other in (cache(heads=4), cache(dim=64), cache(page=128)):
        assert lib.svdq_kv_copy_pages(CACHE, other, AT, 3, None) == EINVAL
    assert lib.svdq_kv_copy_pages(CACHE, CACHE, None, 0, None) == 0
