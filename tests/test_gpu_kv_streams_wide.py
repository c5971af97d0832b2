"""Streams, branches and compaction where calls are wide or odd: many sequences, caches past 4 GB, tables past 64 entries, positions past the rotation's table, norms of one side, the ends of eps,
other streams, captured and replayed calls that share a workspace."""
import numpy as np
import pytest

from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_compact import check
from tests.test_gpu_kv_streams import DEV, Norm, Stream, check_keys, i32

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


def nothing(heads, dim):
    return (np.zeros((0, heads, dim)),) * 2 + (np.zeros((0, heads), int),) * 2


@pytest.mark.parametrize("staged", [False, True])
def test_compaction_of_many_sequences(torch, KV, staged):
    B, rng = 150, np.random.default_rng(1)
    held = rng.integers(1, 90, B)
    kept = np.array([int(rng.integers(0, n + 1)) for n in held])
    first = rng.integers(0, 40, B)
    w = Stream(torch, KV, 2, 64, 32, held, 1, dims=64, positions=200)
    w.append(held)
    d = Stream(torch, KV, 2, 64, 64, first + kept, 2, dims=64, positions=200)
    d.append(first)
    tokens = np.concatenate([rng.permutation(n)[:k] for n, k in zip(held, kept)])
    cu = np.concatenate([[0], np.cumsum(kept)])
    before = [d.rows(b) if first[b] else nothing(2, 64) for b in range(B)]
    moves = KV.KVMoves(i32(torch, cu), i32(torch, tokens), i32(torch, first), i32(torch, w.table), i32(torch, d.table), int(cu[-1]))
    d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=d.cache.compact_workspace(moves) if staged else None)
    torch.cuda.synchronize()
    d.held = first + kept
    for b in rng.permutation(B)[:40].tolist() + [0, 63, 64, 127, 128, B - 1]:
        if kept[b]:
            check(w.rows(b), d.rows(b), first[b], tokens[cu[b]:cu[b + 1]], w.rope_np, False, 2, before[b])


@pytest.mark.parametrize("dim,new,group", [(64, 1, 3), (64, 70, 2), (128, 33, 1)])
def test_streams_of_many_sequences(torch, KV, dim, new, group):
    B, rng = 90, np.random.default_rng(2)
    held = rng.integers(0, 150, B)
    w = Stream(torch, KV, 1, dim, 32, held + new, 3, q_heads=group, dims=dim, norm=dict(first=20))
    w.append(held)
    n = [new if b % 7 else 0 for b in range(B)]
    x, xn, _ = w.append(n)
    w.attend(x, xn, n, window=30, sinks=9)


def test_a_table_of_more_than_64_pages(torch, KV):
    """Old tokens on either side of a table's 64th entry, in one new block."""
    w = Stream(torch, KV, 1, 64, 32, [3000], 4, dims=64)
    w.append([3000])
    d = Stream(torch, KV, 1, 64, 32, [400], 5)
    tokens = np.concatenate([np.arange(2030, 2070), np.arange(0, 3000, 11)])
    moves = KV.KVMoves(i32(torch, [0, len(tokens)]), i32(torch, tokens), i32(torch, [0]), i32(torch, w.table), i32(torch, d.table), len(tokens))
    d.cache.compact(moves, rope=w.rope, source=w.cache)
    d.held = np.array([len(tokens)])
    check(w.rows(0), d.rows(0), 0, tokens, w.rope_np, False, 1, nothing(1, 64))


def test_positions_past_the_table(torch, KV):
    """A table of 50 rows: later positions take its last, in the append, in attention and in compaction."""
    w = Stream(torch, KV, 1, 64, 32, [120], 6, q_heads=2, dims=64, norm={}, positions=50)
    x, xn, _ = w.append([117])
    check_keys(w, [(xn[:, 2:3], xn[:, 3:], np.ones(117, bool))])
    x, xn, _ = w.append([3])
    w.attend(x, xn, [3], window=50, sinks=2)
    d = Stream(torch, KV, 1, 64, 32, [100], 7)
    tokens = np.concatenate([np.arange(0, 120, 3), [118, 119, 49, 50]])
    moves = KV.KVMoves(i32(torch, [0, len(tokens)]), i32(torch, tokens), i32(torch, [40]), i32(torch, w.table), i32(torch, d.table), len(tokens))
    d.append([40])
    before = d.rows(0)
    d.cache.compact(moves, rope=w.rope, source=w.cache)
    d.held = np.array([40 + len(tokens)])
    check(w.rows(0), d.rows(0), 40, tokens, w.rope_np, False, 1, before)


@pytest.mark.parametrize("eps", [1e-30, 1e-6, 1e20])
@pytest.mark.parametrize("sides", ["q", "k", "first", "none"])
def test_norms_of_one_side_and_the_ends_of_eps(torch, KV, eps, sides):
    w = Stream(torch, KV, 2, 128, 64, [200], 8, q_heads=4, dims=64, norm=dict(first=0 if sides != "first" else 70, eps=eps, per_head=True))
    n = w.norm
    for name in ("q", "k", "q_first", "k_first"):
        if not (name[0] == sides or (sides == "first" and name.endswith("first"))):
            setattr(n, name, None)
    up = lambda a: None if a is None else torch.from_numpy(a).to(DEV)
    n.dev = KV.KVNorm(up(n.q), up(n.k), eps, q_first=up(n.q_first), k_first=up(n.k_first), first_tokens=n.first)
    _, xn, _ = w.append([90])
    check_keys(w, [(xn[:, 4:6], xn[:, 6:], np.ones(90, bool))])
    for new in (3, 107):
        x, xn, _ = w.append([new])
        w.attend(x, xn, [new], scale=0.2 if eps < 1 else 1e18)


def test_caches_past_four_gigabytes(torch, KV):
    """Codes of keys, and of values, past 2^32 bytes: append, attention, branches and compaction in the last pages."""
    H, D, P = 8, 128, 64
    pages = (1 << 32) // (H * D * P) + 64      # 4.3 GB of codes each
    w = Stream(torch, KV, H, D, P, [64], 9, q_heads=8, dims=D, norm={}, positions=600)
    w.cache = KV.KVCache(pages, H, D, P)
    refs = torch.ones(pages, dtype=torch.int32, device=DEV)
    refs[3] = refs[5] = 0
    refs[pages - 30:] = 0
    pool = KV.KVPages.from_counts(refs, P)
    table = torch.full((1, 8), -1, dtype=torch.int32, device=DEV)
    w.held = np.array([300])
    x = torch.randn(300, 3 * H, D, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
    step = lambda x, batch: (pool.reserve(w.cache, batch), w.cache.append(x[:, H:2 * H], x[:, 2 * H:], batch, w.rope, norm=w.norm.dev))
    step(x, KV.KVBatch(i32(torch, [0, 300]), i32(torch, [300]), table, 300, 300, 300))
    assert table[0].tolist() == [3, 5, pages - 30, pages - 29, pages - 28, -1, -1, -1]
    few = w.cache      # (reads whole buffers back: of the pages in use only)

    def rows(table, n):
        used = table[0, :(n + P - 1) // P].long()
        w.cache = KV.KVCache.from_buffers(*(t[used].contiguous() for t in (few.k_codes, few.k_scales, few.v_codes, few.v_scales)))
        w.table, w.held = np.arange(len(used))[None], np.array([n])
        got = w.rows(0)
        w.cache = few
        return got
    xn = x.float().cpu().numpy()
    k, v, kb, vb = rows(table, 300)
    y, size = w.norm.ready(xn[:, H:2 * H], np.arange(300), "k", w.rope_np, False)
    assert (np.abs(k - y) <= W.code_bounds(y, W.READY * size, kb[..., None])).all() and (np.abs(v - xn[:, 2 * H:]) <= W.code_bounds(xn[:, 2 * H:], 0.0, vb[..., None])).all()
    # branches
    to, lens = torch.full((2, 8), -1, dtype=torch.int32, device=DEV), i32(torch, [0, 0])
    pool.fork(table, i32(torch, [300]), i32(torch, [0, 0]), to, lens)
    x2 = torch.randn(2, 3 * H, D, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(torch.bfloat16)
    batch = KV.KVBatch(i32(torch, [0, 1, 2]), i32(torch, [301, 301]), to, 2, 1, 301)
    step(x2, batch)
    assert to[:, 4].tolist() == [pages - 27, pages - 26]
    out = w.cache.attention(x2[:, :H], batch, w.rope, norm=w.norm.dev, window=100, sinks=4).float().cpu().numpy()
    x2n = x2.float().cpu().numpy()
    for b in range(2):
        k2, v2, _, _ = rows(to[b:b + 1], 301)
        assert np.array_equal(k2[:256], k[:256]) and np.array_equal(v2[:256], v[:256])
        q, size = w.norm.ready(x2n[b:b + 1, :H], np.array([300]), "q", w.rope_np, False)
        want, tol = W.attention(q, size, k2, v2, [300], np.arange(301), D ** -0.5, True, 100, 4)
        assert (np.abs(out[b:b + 1] - want) <= tol).all()
    # compaction, out of and into such pages
    tokens = np.sort(np.random.default_rng(3).permutation(300)[:130])
    thin = torch.full((1, 8), -1, dtype=torch.int32, device=DEV)
    pool.reserve(w.cache, KV.KVBatch(i32(torch, [0, 130]), i32(torch, [130]), thin, 130, 130, 130))
    assert thin[0, :3].tolist() == [pages - 25, pages - 24, pages - 23]
    moves = KV.KVMoves(i32(torch, [0, 130]), i32(torch, tokens), i32(torch, [0]), table, thin, 130)
    for ws in (None, w.cache.compact_workspace(moves)):
        w.cache.compact(moves, rope=w.rope, workspace=ws)
        check((k, v, kb, vb), rows(thin, 130), 0, tokens, w.rope_np, False, H, nothing(H, D))
    w.cache.copy_pages(i32(torch, [[pages - 30, pages - 1, P], [5, pages - 2, 33]]))
    for t in (few.k_codes, few.k_scales, few.v_codes, few.v_scales):
        assert torch.equal(t[pages - 30], t[pages - 1]) and torch.equal(t[5], t[pages - 2])


def test_calls_on_another_stream_with_memory_of_their_own(torch, KV):
    w = Stream(torch, KV, 2, 128, 64, [400], 10, q_heads=8, dims=128, norm={})
    w.append([300])
    x, xn, _ = w.append([2])
    want = w.attend(x, xn, [2], window=100, sinks=7)
    batch, _ = w.batch([2])
    d = Stream(torch, KV, 2, 128, 64, [200], 11)
    tokens = np.arange(100, 290)
    moves = KV.KVMoves(i32(torch, [0, 190]), i32(torch, tokens), i32(torch, [0]), i32(torch, w.table), i32(torch, d.table), 190)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = w.cache.attention(x[:, :8], batch, w.rope, window=100, sinks=7, norm=w.norm.dev, stream=stream)
    d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=d.cache.compact_workspace(moves, stream=stream), stream=stream)
    stream.synchronize()
    assert np.array_equal(out.float().cpu().numpy().astype(np.float64), want)
    d.held = np.array([190])
    check(w.rows(0), d.rows(0), 0, tokens, w.rope_np, False, 2, nothing(2, 128))


def test_captured_compactions_that_share_a_workspace(torch, KV):
    """Two graphs, one workspace, replayed in turn on one stream with other lists and eager calls between."""
    H, D, P = 2, 128, 64
    w = Stream(torch, KV, H, D, P, [500], 12, dims=D)
    w.append([500])
    old = w.rows(0)
    made, first = [], None
    for seed in (13, 14):
        d = Stream(torch, KV, H, D, P, [300], seed, dims=D)
        tokens = torch.zeros(1, 200, dtype=torch.int32, device=DEV)
        moves = KV.KVMoves(i32(torch, [0, 200]), tokens, i32(torch, [0]), i32(torch, w.table), i32(torch, d.table), 200)
        first = first if first is not None else d.cache.compact_workspace(moves)
        d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=first)      # (loads the kernels)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=first)
        made.append((d, tokens, graph, moves))      # (the graph reads what `moves` holds)
    rng = np.random.default_rng(5)
    for i in range(4):
        lists = []
        for d, tokens, graph, _ in made:
            lists.append(rng.permutation(500)[:200])
            tokens.copy_(i32(torch, lists[-1])[None])
            graph.replay()
        x = torch.ones(1000, device=DEV).cumsum(0)
        torch.cuda.synchronize()
        assert x[-1].item() == 1000
        for (d, *_), chosen in zip(made, lists):
            d.held = np.array([200])
            check(old, d.rows(0), 0, chosen, w.rope_np, False, H, nothing(H, D))


def test_nothing_to_do(torch, KV):
    w = Stream(torch, KV, 2, 64, 32, [64], 15)
    keep = [t.clone() for t in w.buffers()]
    empty = i32(torch, np.zeros(0))
    moves = KV.KVMoves(i32(torch, [0]), empty, empty, i32(torch, np.zeros((0, 2))), i32(torch, np.zeros((0, 2))), 0)
    w.cache.compact(moves, workspace=w.cache.compact_workspace(moves))
    moves = KV.KVMoves(i32(torch, [0, 0]), empty, i32(torch, [5]), i32(torch, w.table), i32(torch, w.table), 0)
    w.cache.compact(moves)
    pool = KV.KVPages(4, 32)
    none = i32(torch, np.zeros((0, 2)))
    pool.release(none)
    pool.fork(none, empty, empty, none, empty)
    rows = torch.full((2, 2), 3, dtype=torch.int32, device=DEV)
    lens = i32(torch, [7, 7])
    pool.fork(none, empty, i32(torch, [0, 1]), rows, lens)      # no parents
    torch.cuda.synchronize()
    assert (rows == -1).all() and (lens == 0).all() and not pool.refs.any()
    assert all(torch.equal(a, b) for a, b in zip(keep, w.buffers()))
    with pytest.raises(S.SvdqError):
        pool.fork(rows, lens, i32(torch, [0, 0]), rows, i32(torch, [0, 0]))      # the tables overlap
