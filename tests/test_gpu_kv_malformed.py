"""Counts of tokens that do not ascend or leave their range: every call does what the calls with the counts that are left would do, sequence by sequence, and touches nothing else.  The pool
on another stream, with what it reads and writes kept till that stream is done."""
import numpy as np
import pytest

from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_pages import Pool, empty
from tests.test_gpu_kv_streams import DEV, Stream, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "these tests need the MI355X"
    S.lib()
    return t


@pytest.fixture(scope="module")
def KV(torch):
    from paper_2411_05007_amd import kv
    return kv


def ranges(cu, total):
    """(first, count) of each sequence, as far as cu ascends within 0 .. total"""
    got = []
    for a, b in zip(cu, cu[1:]):
        a = min(max(a, 0), total)
        got.append((a, min(max(b, a), total) - a))
    return got


@pytest.mark.parametrize("cu", [[0, 60, 20], [5, 200, 90], [-9, -3, 400], [80, 80, 80], [40, 0, 80]])
@pytest.mark.parametrize("first", [[0, 5], [-7, 60], [-2 ** 31, 2 ** 31 - 1], [33, 31]])
def test_moves_that_are_malformed(torch, KV, cu, first):
    w = Stream(torch, KV, 2, 64, 32, [64, 64], 37)
    w.append([64, 64])
    tokens = np.tile(np.arange(40), 2)
    seen = []
    for way in ("direct", "staged", "one by one"):
        d = Stream(torch, KV, 2, 64, 32, [64, 64], 38)
        d.append([40, 40])      # (blocks that hold tokens already)
        keep = [t.clone() for t in d.buffers()]
        if way == "one by one":
            for b, (at, n) in enumerate(ranges(cu, 80)):
                moves = KV.KVMoves(i32(torch, [0, n]), i32(torch, tokens[at:at + n]), i32(torch, [max(first[b], 0)]), i32(torch, w.table[b:b + 1]), i32(torch, d.table[b:b + 1]), n)
                d.cache.compact(moves, source=w.cache)
                torch.cuda.synchronize()
        else:
            moves = KV.KVMoves(i32(torch, cu), i32(torch, tokens), i32(torch, first), i32(torch, w.table), i32(torch, d.table), 80)
            d.cache.compact(moves, source=w.cache, workspace=d.cache.compact_workspace(moves) if way == "staged" else None)
            torch.cuda.synchronize()
        spare = sorted(set(range(d.pages)) - set(d.table.ravel().tolist()))
        assert spare and all(torch.equal(a[spare], b[spare]) for a, b in zip(keep, d.buffers()))
        seen.append([t.cpu().numpy() for t in d.buffers()])
    k, ks, v, vs = zip(*seen)
    for i in (1, 2):
        assert np.array_equal(ks[0], ks[i]) and np.array_equal(vs[0], vs[i]) and np.array_equal(v[0], v[i])
        assert np.array_equal(k[0], k[i])


@pytest.mark.parametrize("cu", [[0, 60, 20, 20, 90], [-5, 400, 7, 8, 9], [90, 0, 90, 0, 90], [0, 0, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 30, 60, 2 ** 31 - 1]])
def test_reservations_that_are_malformed(torch, KV, cu):
    w = Pool(torch, KV, 12, 32)
    dev, host = empty(torch, 4, 3)
    w.reserve(dev, host, [20, 64, 5, 33], [20, 64, 5, 33])
    to, ho = empty(torch, 4, 3)
    out, hl = i32(torch, [0] * 4), [0] * 4
    parents = [0, 1, 1, 3]
    w.pool.fork(dev, i32(torch, [20, 64, 5, 33]), i32(torch, parents), to, out)
    w.model.fork(host, [20, 64, 5, 33], parents, ho, hl)
    lens = [30, 70, 64, 96]
    missing = i32(torch, [77])
    w.pool.reserve(w.caches[0], KV.KVBatch(i32(torch, cu), i32(torch, lens), to, 90, 90, 96), missing)
    copies, lacks = w.model.reserve(ho, [n for _, n in ranges(cu, 90)], lens)
    for g, page, tokens in copies:
        if g >= 0:
            for x in w.shadow[0]:
                x[page, :, :(tokens + 31) // 32] = x[g, :, :(tokens + 31) // 32]
    w.check((dev, host), (to, ho))
    assert missing.tolist() == [lacks]
    assert w.model.refs == np.bincount([g for h in (host, ho) for row in h for g in row if g >= 0], minlength=12).tolist()


def test_the_pool_on_another_stream_with_what_it_needs_kept(torch, KV):
    """The current stream is kept busy, and reads what the other one wrote only when that is done."""
    w = Pool(torch, KV, 40, 64)
    dev, host = empty(torch, 3, 6)
    to, ho = empty(torch, 4, 6)
    lens, parent, out, hl = i32(torch, [100, 5, 0]), i32(torch, [0, 0, 1, 2]), i32(torch, [0] * 4), [0] * 4
    first = KV.KVBatch(i32(torch, [0, 100, 105, 105]), lens, dev, 105, 100, 100)
    steps = i32(torch, [30, 1, 2, 3])
    second = KV.KVBatch(i32(torch, [0, 30, 31, 33, 36]), out, to, 36, 30, 200)
    missing = [i32(torch, [77]) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    busy = torch.zeros(1 << 24, device=DEV)
    for _ in range(20):
        busy.add_(1.0)
    w.pool.reserve(w.caches[0], first, missing[0], stream=stream)
    w.pool.fork(dev, lens, parent, to, out, stream=stream)
    with torch.cuda.stream(stream):
        out.add_(steps)
    w.pool.reserve(w.caches[0], second, missing[1], stream=stream)
    stream.synchronize()
    w.model.reserve(host, [100, 5, 0], [100, 5, 0])
    w.model.fork(host, [100, 5, 0], [0, 0, 1, 2], ho, hl)
    hl = [a + b for a, b in zip(hl, [30, 1, 2, 3])]
    copies, lacks = w.model.reserve(ho, [30, 1, 2, 3], hl)
    for g, page, tokens in copies:
        if g >= 0:
            for x in w.shadow[0]:
                x[page, :, :(tokens + 31) // 32] = x[g, :, :(tokens + 31) // 32]
    w.check((dev, host), (to, ho))
    assert [m.item() for m in missing] == [0, lacks] and out.tolist() == hl and busy[0].item() == 20
    w.pool.release(to, stream=stream)
    w.model.release(ho)
    stream.synchronize()
    w.check((dev, host), (to, ho))
