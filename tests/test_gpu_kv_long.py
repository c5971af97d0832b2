"""Attention over the paged 8-bit cache at the sizes where the kernels of many rows, the parts of their keys and the cut keys of few rows take over; batches of
more sequences than a wavefront has lanes; appends that take several heads a workgroup.  The cache is a pool of pages that sequences share at random, its content
is read back by gather (which has tests of its own, bit for bit), and rows are sampled where tiles, sequences and masks begin and end."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from paper_2411_05007_amd import svdq as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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


def i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Pool:
    """Pages with random content: blocks of different scales, some channels louder."""

    def __init__(self, torch, KV, heads, dim, page, pages, seed, nan_pages=()):
        self.torch, self.KV, self.heads, self.dim, self.page, self.pages = torch, KV, heads, dim, page, pages
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        n = pages * page
        x = torch.randn(n, 2 * heads, dim, generator=gen, device=DEV)
        x *= torch.exp2(torch.randint(-2, 3, (n // 32, 2 * heads, 1), generator=gen, device=DEV).float()).repeat_interleave(32, 0)
        for p in nan_pages:
            x[p * page + 3, heads - 1, 5] = float("nan")      # a key of the last head
        x = x.to(torch.bfloat16)
        self.cache = KV.KVCache(pages, heads, dim, page)
        order = torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous()
        self.cache.append(x[:, :heads], x[:, heads:], KV.KVBatch(i32(torch, [0, n]), i32(torch, [n]), order, n, n, n))

    def rows(self, table, length, head):
        """keys and values fp64 [length, 1, dim] of a head"""
        t = self.torch.from_numpy(np.ascontiguousarray(table[None])).to(DEV)
        k, v = self.cache.gather(self.KV.KVRows(i32(self.torch, [0]), i32(self.torch, [0, length]), t, length))
        return [x[:, head:head + 1].double().cpu().numpy() for x in (k, v)]


def check(torch, KV, pool, rng, group, table, lens, new, causal, window, rope=None, max_len=None, extra=0, samples=40, want_nan=False, scale=None):
    """Attention of new[b] tokens at the end of lens[b]; `extra` tokens behind them belong to no sequence."""
    H, D, page = pool.heads, pool.dim, pool.page
    B, Q = len(lens), H * group
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1]) + extra
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(rng.integers(1 << 30)))
    q = torch.randn(T, Q + 3, D, generator=gen, device=DEV).to(torch.bfloat16)[:, 1:Q + 1]
    batch = KV.KVBatch(i32(torch, cu), i32(torch, lens), i32(torch, table), T, max(new), max_len or max(lens))
    n = pool.cache.attention_workspace(batch, Q).numel()
    outs = []
    for fill in (0xFF, 0x33):
        ws = torch.full((n + 256,), fill, dtype=torch.uint8, device=DEV)
        out = torch.full((T + 2, Q, D), 7.0, dtype=torch.bfloat16, device=DEV)
        pool.cache.attention(q, batch, rope and rope[1], causal=causal, window=window, out=out[1:-1], workspace=ws[:n], scale=scale)
        torch.cuda.synchronize()
        assert bool((ws[n:] == fill).all()) and bool((out[0] == 7).all()) and bool((out[T + 1 - extra:] == 7).all())
        outs.append(out[1:-1])
    assert torch.equal(outs[0].view(torch.int16), outs[1].view(torch.int16))      # (whatever the workspace held)
    got, qn = outs[0], q.float()
    # rows where something begins or ends, and some anywhere
    picks = set()
    for b in sorted({0, B - 1} | set(int(x) for x in rng.integers(0, B, 6))):
        if new[b] == 0:
            continue
        edge = [0, new[b] - 1, 31 // group, 32 // group, 127 // group, 128 // group, 255 // group, 256 // group]
        picks |= {(b, int(i)) for i in edge + list(rng.integers(0, new[b], 3)) if 0 <= i < new[b]}
    picks = sorted(picks)
    if len(picks) > samples:
        picks = [picks[i] for i in sorted(rng.choice(len(picks), samples, replace=False))]
    memo, nans, checked = {}, 0, 0
    for b, i in picks:
        pos = lens[b] - new[b] + i
        hi = min(lens[b], pos + 1) if causal else lens[b]
        lo = max(0, pos + 1 - window) if causal and window else 0
        keys = np.arange(lo, max(lo, hi))
        place = table[b, keys // page]
        keys = keys[(place >= 0) & (place < pool.pages)]
        for h in {int(rng.integers(H)), H - 1}:
            if (b, h) not in memo:
                memo[b, h] = pool.rows(table[b], max(lens[b], 1), h)
            k, v = memo[b, h]
            x = qn[cu[b] + i, h * group:(h + 1) * group].cpu().numpy()
            x = K.rotate(x, max(pos, 0), rope[0], rope[2])[None].astype(np.float64) if rope else x[None].astype(np.float64)
            want, tol = K.attention(x, k[keys], v[keys], [0], D ** -0.5 if scale is None else scale, False, 0) if keys.size else (np.zeros((1, group, D)),) * 2
            g = got[cu[b] + i, h * group:(h + 1) * group].double().cpu().numpy()[None]
            assert np.array_equal(np.isnan(g), np.isnan(want)), (b, i, h)
            nans += int(np.isnan(want).any())
            ok = ~np.isnan(want)
            off = (np.abs(g - want) - tol)[ok]
            assert off.size == 0 or off.max() <= 0, (b, i, h, float(off.max()))
            checked += 1
    assert checked > 0 and (nans > 0) == want_nan
    return got


def shared(rng, pool, lens, holes=False):
    width = max(1, (max(lens) + pool.page - 1) // pool.page)
    table = rng.integers(0, pool.pages, (len(lens), width)).astype(np.int32)
    if holes:
        out = rng.random(table.shape)
        table[out < 0.1] = -1
        table[out > 0.9] = pool.pages + 5
    return table


def turn(torch, KV, positions, dims, interleaved):
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(dims // 2) * 2.0 / dims)
    t = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
    return t, KV.Rope(torch.from_numpy(t).to(DEV), interleaved), interleaved


@pytest.mark.parametrize("new,length,causal", [(256, 4200, True), (256, 4097, False), (300, 4352, True)])
def test_even_batches_of_long_sequences(torch, KV, new, length, causal):
    rng = np.random.default_rng(new + length)
    pool = Pool(torch, KV, 8, 128, 64, 90, 1)
    lens = [length] * 32
    check(torch, KV, pool, rng, 1, shared(rng, pool, lens), lens, [new] * 32, causal, 0, turn(torch, KV, length, 128, False))


def test_even_batches_of_whole_prompts(torch, KV):
    rng = np.random.default_rng(5)
    pool = Pool(torch, KV, 4, 128, 128, 40, 2)
    lens = [4100] * 4      # the first rows see one tile, the last all
    check(torch, KV, pool, rng, 2, shared(rng, pool, lens), lens, [4100] * 4, True, 0)


@pytest.mark.parametrize("dim,page,heads,group,causal,window,holes", [
    (128, 64, 8, 2, True, 0, False), (128, 64, 8, 2, True, 300, False), (128, 32, 8, 2, False, 0, True), (128, 256, 8, 3, True, 0, True),
    (64, 64, 12, 1, True, 0, False), (64, 32, 12, 1, True, 65, True), (64, 128, 6, 5, False, 0, False),
    (256, 64, 2, 4, True, 0, False), (256, 32, 2, 4, True, 1000, True),
])
def test_ragged_batches_of_many_rows(torch, KV, dim, page, heads, group, causal, window, holes):
    rng = np.random.default_rng(dim + page + group + window)
    B = 40 if dim == 256 else 24
    new = [int(n) for n in rng.integers(1, 200 * 2 // group if group < 3 else 200, B)]
    new[0], new[3], new[B - 1] = max(new), 0, 1
    lens = [n + int(h) for n, h in zip(new, rng.integers(0, 2600, B))]
    lens[0], lens[1] = 2600 + new[0], new[1]
    pool = Pool(torch, KV, heads, dim, page, 3000 // page + 20, dim + page)
    check(torch, KV, pool, rng, group, shared(rng, pool, lens, holes), lens, new, causal, window, turn(torch, KV, 1000, dim // 2, group % 2 == 1))


@pytest.mark.parametrize("dim,heads,group,new,lens,causal,window,extra", [
    (128, 2, 4, [300, 37], [8000, 900], True, 0, 0),                   # few row tiles on many keys
    (128, 2, 4, [300, 37], [8000, 37], True, 2990, 5),
    (128, 2, 4, [37, 300, 0], [8001, 300, 0], False, 0, 0),
    (128, 1, 8, [2000], [2000], True, 0, 3),                           # parts without a key
    (64, 3, 4, [700, 650], [12000, 11111], True, 0, 0),
    (256, 2, 2, [600] * 6, [3000, 2999, 600, 3000, 2048, 1100], True, 0, 7),
])
@pytest.mark.parametrize("holes", [False, True])
def test_keys_in_parts(torch, KV, dim, heads, group, new, lens, causal, window, extra, holes):
    rng = np.random.default_rng(dim + len(new) + window)
    pool = Pool(torch, KV, heads, dim, 64, 140, 7)
    check(torch, KV, pool, rng, group, shared(rng, pool, lens, holes), lens, new, causal, window, turn(torch, KV, max(lens), dim, True), extra=extra)


@pytest.mark.parametrize("dim,heads,group,new,lens,causal,window,extra", [
    (128, 2, 4, [300, 1, 4, 5, 0, 1], [8000, 7000, 4, 900, 0, 1], True, 0, 0),        # with parts of the chunk's keys; 16 rows and 20
    (128, 8, 4, [1] * 20 + [512] + [2] * 11, [8000] * 20 + [512] + [777] * 11, True, 0, 4),
    (64, 3, 8, [1, 2, 3, 700, 1], [12000, 5000, 40, 12000, 1], True, 500, 0),
    (64, 12, 1, [400, 16, 17, 1, 399, 15, 1, 1], [3000, 16, 2000, 3000, 399, 64, 65, 1], False, 0, 0),
    (256, 2, 2, [600, 1, 8, 9, 1], [3000, 2999, 600, 3000, 33], True, 0, 2),
    (128, 2, 17, [300, 1, 1, 8], [8000, 7999, 5, 64], True, 0, 0),                       # a single token is two tiles of rows
    # the single tokens in a launch of their own
    (64, 12, 1, [400] + [16] * 20 + [17] * 2 + [1] * 40, [3000] + [2900, 16] * 10 + [17, 1700] + [1, 3000, 33, 640] * 10, True, 0, 3),
    (256, 2, 2, [1] * 15 + [600] + [1] * 15 + [8, 9], [2999, 1, 700] * 5 + [3000] + [64, 2048, 33] * 5 + [8, 2000], True, 0, 0),
    (128, 8, 8, [1] * 30 + [700], [9000, 1, 3100] * 10 + [8999], True, 3000, 0),
    (128, 8, 4, [512, 1], [4000, 100000], True, 0, 0),
])
@pytest.mark.parametrize("holes", [False, True])
def test_chunks_beside_single_tokens(torch, KV, dim, heads, group, new, lens, causal, window, extra, holes):
    rng = np.random.default_rng(dim + len(new))
    pool = Pool(torch, KV, heads, dim, 64, 140, 27)
    check(torch, KV, pool, rng, group, shared(rng, pool, lens, holes), lens, new, causal, window, turn(torch, KV, max(lens), dim // 2, False), extra=extra, samples=60)


@pytest.mark.parametrize("heads,group,new,length", [(8, 1, 256, 4200), (8, 2, 150, 2000), (2, 4, 300, 8000)])
def test_a_key_that_is_not_finite_reaches_the_rows_that_see_it(torch, KV, heads, group, new, length):
    rng = np.random.default_rng(heads + new)
    B = 32 if heads == 8 else 2
    pool = Pool(torch, KV, heads, 128, 64, 100, 11, nan_pages=(0,))
    lens = [length] * B
    table = rng.integers(1, pool.pages, (B, (length + 63) // 64)).astype(np.int32)
    table[0, (length - new // 2) // 64] = 0      # some of the new tokens of the first sequence see it
    check(torch, KV, pool, rng, group, table, lens, [new] * B, True, 0, want_nan=True)


def test_long_negative_and_zero_scales(torch, KV):
    rng = np.random.default_rng(21)
    pool = Pool(torch, KV, 4, 128, 64, 60, 13)
    lens = [3000] * 16
    table = shared(rng, pool, lens)
    for scale in (-0.05, 0.0, 0.5):
        check(torch, KV, pool, rng, 2, table, lens, [200] * 16, True, 0, samples=15, scale=scale)


@pytest.mark.parametrize("B,heads,group,most,length,window", [(200, 4, 2, 3, 500, 0), (150, 4, 2, 60, 600, 0), (130, 4, 3, 50, 900, 100), (65, 1, 1, 1, 3000, 0)])
def test_more_sequences_than_lanes(torch, KV, B, heads, group, most, length, window):
    rng = np.random.default_rng(B)
    new = [int(n) for n in rng.integers(0, most + 1, B)]
    new[0] = most
    lens = [n + int(h) for n, h in zip(new, rng.integers(0, length, B))]
    pool = Pool(torch, KV, heads, 128, 32, 50, 17)
    check(torch, KV, pool, rng, group, shared(rng, pool, lens, True), lens, new, True, window, samples=60)


@pytest.mark.parametrize("dim,heads,group,new,length,window", [(64, 1, 4, 1, 2201600, 0), (64, 1, 17, 1, 1433600, 0), (128, 1, 8, 2, 614400, 0)])
def test_very_long_sequences(torch, KV, dim, heads, group, new, length, window):
    """The table repeats a pool of ten pages: the softmax over all keys is that over one round of them."""
    rng = np.random.default_rng(group)
    page, pages = 1024, 10
    pool = Pool(torch, KV, heads, dim, page, pages, 19)
    table = np.tile(np.arange(pages, dtype=np.int32), length // (page * pages))[None]
    T, Q = new, heads * group
    q = torch.from_numpy(rng.standard_normal((T, Q, dim))).to(DEV).to(torch.bfloat16)
    batch = KV.KVBatch(i32(torch, [0, T]), i32(torch, [length]), i32(torch, table), T, T, length)
    got = pool.cache.attention(q, batch, causal=False).double().cpu().numpy()
    k, v = pool.rows(table[0], page * pages, 0)
    want, tol = K.attention(q.double().cpu().numpy(), k, v, np.zeros(T), dim ** -0.5, False, 0)
    tol += (length - page * pages) * 2.0 ** -33 * np.abs(v).max()
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("new,bound", [(1, 900), (3, 32), (60, 900), (300, 700)])
def test_lengths_far_past_the_bound(torch, KV, new, bound):
    rng = np.random.default_rng(new)
    pool = Pool(torch, KV, 2, 128, 64, 100, 23)
    lens = [20000, 9000, new]
    check(torch, KV, pool, rng, 4, shared(rng, pool, lens), lens, [new] * 3, True, 0, max_len=bound, samples=15)


def test_memory_that_a_call_allocates_for_another_stream_stays_its_own(torch, KV):
    """The workspace is the binding's, on the current stream; its next owner there must not write to it while the call's stream is still to run."""
    rng = np.random.default_rng(4)
    pool = Pool(torch, KV, 2, 128, 64, 60, 29)
    lens = [9000, 5000]
    table = i32(torch, shared(rng, pool, lens))
    q = torch.randn(2, 8, 128, device=DEV).to(torch.bfloat16)
    batch = KV.KVBatch(i32(torch, [0, 1, 2]), i32(torch, lens), table, 2, 1, 9000)
    want = pool.cache.attention(q, batch)
    n = pool.cache.attention_workspace(batch, 8).numel()
    assert n > 4096      # (parts that meet)
    rows = KV.KVRows(i32(torch, [0]), i32(torch, [0, 9000]), table[:1].contiguous(), 9000)
    kv = pool.cache.gather(rows)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device=DEV)
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(4):
                big @ big      # (the side stream is busy for a while)
        got = pool.cache.attention(q, batch, stream=side)
        mine = [torch.full((n,), 0x41, dtype=torch.uint8, device=DEV) for _ in range(4)]
        k, v = pool.cache.gather(rows, stream=side)
        mine += [torch.full((9000, 2, 128), 3.0, dtype=torch.bfloat16, device=DEV) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(k, kv[0]) and torch.equal(v, kv[1])
        del got, k, v, mine


# ---- append and gather ----------------------------------------------------------------------------------------------------------------------


def bytes_of(cache):
    return [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


@pytest.mark.parametrize("dim,heads,held,tokens", [(64, 42, 0, 4000), (64, 41, 37, 3990), (128, 19, 5, 9000), (256, 10, 33, 16000), (128, 13, 1, 6000)])
def test_heads_together_are_as_heads_alone(torch, KV, dim, heads, held, tokens):
    """Many tokens: a workgroup takes several heads.  One head at a time, each in a cache of its own, gives the same bytes."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(dim + heads)
    total = held + tokens
    pages = (total + 63) // 64
    x = torch.randn(total, 2 * heads, dim, generator=gen, device=DEV)
    x *= torch.exp2(torch.randint(-3, 4, (total, 2 * heads, 1), generator=gen, device=DEV).float())
    x[held + 100, 3, 1] = float("inf")
    x[held + 70, heads + 2, 0] = float("nan")
    x = x.to(torch.bfloat16)
    table = torch.randperm(pages, generator=gen, device=DEV).int()[None].contiguous()
    _, rope, _ = turn(torch, KV, total, dim, True)

    def fill(cache, k, v):
        for a, b in ((0, held), (held, total)):
            if b > a:
                cache.append(k[a:b], v[a:b], KV.KVBatch(i32(torch, [0, b - a]), i32(torch, [b]), table, b - a, b - a, b), rope)
        return bytes_of(cache)
    together = fill(KV.KVCache(pages, heads, dim, 64), x[:, :heads], x[:, heads:])
    for h in range(heads):
        alone = fill(KV.KVCache(pages, 1, dim, 64), x[:, h:h + 1], x[:, heads + h:heads + h + 1])
        for a, b in zip(together, alone):
            assert torch.equal(a[:, h], b[:, 0]), h


def test_append_and_gather_of_many_sequences_are_as_one_by_one(torch, KV):
    rng = np.random.default_rng(3)
    B, heads, dim, page = 150, 3, 64, 32
    held, new = rng.integers(0, 90, B), rng.integers(0, 40, B)
    new[0], new[7], new[B - 1] = 0, 39, 1
    width = 5
    pages = B * width
    table = rng.permutation(pages).reshape(B, width).astype(np.int32)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    caches = [KV.KVCache(pages, heads, dim, page) for _ in range(2)]
    for before, count in ((np.zeros(B, int), held), (held, new)):
        cu = np.concatenate([[0], np.cumsum(count)])
        x = torch.randn(int(cu[-1]), 2 * heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
        caches[0].append(x[:, :heads], x[:, heads:], KV.KVBatch(i32(torch, cu), i32(torch, before + count), i32(torch, table), int(cu[-1]), int(count.max()), 130))
        for b in range(B):
            n = int(count[b])
            if n:
                y = x[cu[b]:cu[b + 1]]
                caches[1].append(y[:, :heads], y[:, heads:], KV.KVBatch(i32(torch, [0, n]), i32(torch, [before[b] + n]), i32(torch, table[b:b + 1]), n, n, 130))
        assert all(torch.equal(a, b) for a, b in zip(bytes_of(caches[0]), bytes_of(caches[1])))
    first = rng.integers(0, 20, B)
    count = np.maximum(0, held + new - first)
    cu = np.concatenate([[0], np.cumsum(count)])
    got = caches[0].gather(KV.KVRows(i32(torch, first), i32(torch, cu), i32(torch, table), int(cu[-1])))
    for b in range(0, B, 7):
        one = caches[0].gather(KV.KVRows(i32(torch, first[b:b + 1]), i32(torch, [0, count[b]]), i32(torch, table[b:b + 1]), int(count[b])))
        assert all(torch.equal(g[cu[b]:cu[b + 1]], o) for g, o in zip(got, one))


def test_strides_the_entry_points_refuse(torch, KV):
    cache = KV.KVCache(2, 1, 64, 32)
    batch = KV.KVBatch(i32(torch, [0, 1]), i32(torch, [1]), i32(torch, [[0]]), 1, 1, 1)
    x = torch.zeros(64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(S.SvdqError, match="unsupported"):
        cache.append(torch.as_strided(x, (1, 1, 64), ((1 << 25) + 8, 64, 1)), torch.as_strided(x, (1, 1, 64), (64, 64, 1)), batch)


def test_workspaces_that_are_refused(torch, KV):
    cache = KV.KVCache(2, 1, 64, 32)
    batch = KV.KVBatch(i32(torch, [0, 1]), i32(torch, [1]), i32(torch, [[0]]), 1, 1, 1)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device=DEV)
    for bad in (torch.zeros(256, dtype=torch.uint8), torch.zeros(64, dtype=torch.float32, device=DEV), torch.zeros(512, dtype=torch.uint8, device=DEV)[::2]):
        with pytest.raises(AssertionError):
            cache.attention(q, batch, workspace=bad)
    for bad in (torch.zeros(128, dtype=torch.uint8, device=DEV), torch.zeros(1024, dtype=torch.uint8, device=DEV)[16:]):
        with pytest.raises(S.SvdqError):
            cache.attention(q, batch, workspace=bad)
