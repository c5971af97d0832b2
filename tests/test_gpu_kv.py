"""The paged 8-bit cache of keys and values on the GPU: codes and scale bytes bit for bit against the oracle, attention within what its roundings
allow (oracle/kv_oracle.py derives that per output), over head layouts, ragged and empty sequences, strides, garbage in unused places."""
import os

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


class World:
    """Sequences with a cache on the GPU, filled with bytes that must not matter, and the oracle's beside it."""

    def __init__(self, torch, KV, heads, dim, page, capacity, seed, q_heads=None, dims=None, interleaved=False, gain=1.0, positions=None, fill=0xFF):
        self.torch, self.KV, self.rng = torch, KV, np.random.default_rng(seed)
        self.heads, self.dim, self.page, self.q_heads, self.gain = heads, dim, page, q_heads or heads, gain
        B = len(capacity)
        width = max(1, max((c + page - 1) // page for c in capacity))
        self.pages = B * width + 3
        order = self.rng.permutation(self.pages)
        self.table = np.full((B, width), -1, np.int32)
        at = 0
        for b, c in enumerate(capacity):
            n = (c + page - 1) // page
            self.table[b, :n] = order[at:at + n]
            at += n
        self.cache = KV.KVCache(self.pages, heads, dim, page)
        for t in (self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales):
            t.fill_(fill)
        self.held = [0] * B
        self.oracle = K.Cache(heads, dim)
        self.rope_np, self.rope, self.interleaved = None, None, interleaved
        if dims:
            n = positions or max(capacity) + 1
            a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(dims // 2) * 2.0 / dims)
            self.rope_np = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
            self.rope = KV.Rope(torch.from_numpy(self.rope_np).to(DEV), interleaved)

    def i32(self, x):
        return self.torch.tensor(np.asarray(x), dtype=self.torch.int32, device=DEV)

    def rows(self, T, scale=1.0):
        """qkv of T tokens as a QKV layer leaves it: bf16 on the GPU and fp32 in numpy"""
        x = self.rng.standard_normal((T, self.q_heads + 2 * self.heads, self.dim)) * self.gain * scale
        t = self.torch.from_numpy(x).to(DEV).to(self.torch.bfloat16)
        return t, t.float().cpu().numpy()

    def batch(self, new):
        cu = np.concatenate([[0], np.cumsum(new)])
        lens = [h + n for h, n in zip(self.held, new)]
        return self.KV.KVBatch(self.i32(cu), self.i32(lens), self.i32(self.table), int(cu[-1]), max(new), max(lens)), cu

    def append(self, new, scale=1.0, poke=None):
        batch, cu = self.batch(new)
        x, xn = self.rows(int(cu[-1]), scale)
        if poke is not None:
            poke(x)
            xn = x.float().cpu().numpy()
        H, Q = self.heads, self.q_heads
        self.cache.append(x[:, Q:Q + H], x[:, Q + H:], batch, self.rope)
        before = list(self.held)
        for b, n in enumerate(new):
            s = xn[cu[b]:cu[b + 1]]
            self.oracle.append(b, self.held[b], s[:, Q:Q + H], s[:, Q + H:], self.rope_np, self.interleaved)
            self.held[b] += n
        self.torch.cuda.synchronize()
        return x, xn, cu, before

    def check_cache(self):
        kc, ks, vc, vs = (t.cpu().numpy() for t in (self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales))
        for b, n in enumerate(self.held):
            for blk in range((n + 31) // 32):
                page, at, live = self.table[b, blk * 32 // self.page], blk * 32 % self.page // 32, min(32, n - 32 * blk)
                for h in range(self.heads):
                    k, v = K.block_numbers(kc[page, h, at], vc[page, h, at])
                    kb, kn = self.oracle.k[b, blk]
                    vb, vn = self.oracle.v[b, blk]
                    assert (ks[page, h, at], vs[page, h, at]) == (kb[h], vb[h]), (b, blk, h)
                    assert np.array_equal(k[:live], kn[h, :live], equal_nan=True) and np.array_equal(v[:live], vn[h, :live]), (b, blk, h)
        used = {int(p) for b, n in enumerate(self.held) for p in self.table[b, :(n + self.page - 1) // self.page]}
        for p in set(range(self.pages)) - used:
            assert all((t[p] == 0xFF).all() for t in (kc, ks, vc, vs)), "a page of no sequence was written"

    def attend(self, x, xn, new, before, causal=True, window=0, scale=None, **kw):
        batch, cu = self.batch(new)      # (held counts the new tokens already)
        batch = self.KV.KVBatch(batch.cu_new, self.i32(self.held), batch.block_table, batch.new_tokens, max(new), max(self.held))
        out = self.torch.full((int(cu[-1]), self.q_heads, self.dim), 7.0, dtype=self.torch.bfloat16, device=DEV)
        got = self.cache.attention(x[:, :self.q_heads], batch, self.rope, scale=scale, causal=causal, window=window, out=out, **kw)
        self.torch.cuda.synchronize()
        got = got.float().cpu().numpy().astype(np.float64)
        for b, n in enumerate(new):
            if n == 0:
                continue
            k, v = self.oracle.rows(b, 0, self.held[b])
            q = np.stack([K.rotate(xn[cu[b] + i, :self.q_heads], before[b] + i, self.rope_np, self.interleaved) for i in range(n)]).astype(np.float64)
            want, tol = K.attention(q, k, v, before[b] + np.arange(n), self.dim ** -0.5 if scale is None else scale, causal, window)
            g = got[cu[b]:cu[b + 1]]
            assert np.array_equal(np.isnan(g), np.isnan(want)), b
            ok = ~np.isnan(want)
            off = np.abs(g - want)[ok] - tol[ok]
            assert off.size == 0 or off.max() <= 0, (b, off.max(), np.unravel_index(np.argmax(np.where(ok, np.abs(g - want) - tol, -1)), g.shape))
        return got


# ---- append and gather ---------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,heads,page,dims,inter,steps", [
    (128, 2, 64, 128, False, [[70, 1, 33, 0]] + [[1, 1, 1, 1]] * 3),
    (128, 3, 32, 64, True, [[31, 32, 1], [2, 33, 0], [0, 1, 64]]),
    (64, 5, 128, 64, False, [[129, 5], [1, 27], [1, 1]]),
    (64, 1, 64, 32, True, [[1], [1], [30], [1], [40]]),
    (64, 2, 64, 0, False, [[3, 0, 65], [64, 1, 2]]),
    (256, 2, 64, 256, False, [[40, 3], [1, 62]]),
    (256, 1, 1024, 96, True, [[37], [1]]),
])
def test_append_fills_blocks_as_the_oracle_does(torch, KV, dim, heads, page, dims, inter, steps):
    w = World(torch, KV, heads, dim, page, np.sum(steps, axis=0), 10 + dim + heads, q_heads=2 * heads, dims=dims, interleaved=inter)
    for i, new in enumerate(steps):      # later tokens are larger or smaller: scales grow, or stay
        w.append(new, scale=[1.0, 3.7, 0.2, 40.0, 1e-3][i % 5])
        w.check_cache()


@pytest.mark.parametrize("scale", [1e-36, 1e-30, 1e30, 0.0])
def test_append_at_the_ends_of_the_range(torch, KV, scale):
    w = World(torch, KV, 2, 64, 32, [50], 3)
    w.append([20], scale=scale)
    w.check_cache()
    w.append([30], scale=1.0)
    w.check_cache()


def test_append_again_gives_the_same_bytes(torch, KV):
    w = World(torch, KV, 2, 128, 64, [100, 40], 4, dims=128)
    w.append([45, 7])
    batch, cu = w.batch([50, 33])
    x, _ = w.rows(83, 5.0)
    got = []
    for _ in range(2):
        w.cache.append(x[:, 2:4], x[:, 4:], batch, w.rope)
        got.append([t.clone() for t in (w.cache.k_codes, w.cache.v_codes, w.cache.k_scales, w.cache.v_scales)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_vectors_that_are_not_finite_are_kept_apart(torch, KV, value):
    w = World(torch, KV, 2, 64, 32, [90], 5, q_heads=4)

    def poke(x):
        x[3, 4, 7] = value       # key of head 0, token 3
        x[40, 7, 0] = value      # value of head 1, token 40
    x, xn, cu, before = w.append([70], poke=poke)
    w.check_cache()
    w.attend(x, xn, [70], before)                       # NaN where the token is seen, and nowhere else
    x, xn, cu, before = w.append([20], scale=30.0)      # the scales grow: NaN stays
    w.check_cache()
    w.attend(x, xn, [20], before, window=9)             # past both
    w.attend(x, xn, [20], before)


def test_tables_and_lengths_out_of_range_touch_nothing(torch, KV):
    w = World(torch, KV, 2, 64, 32, [64, 64], 6, fill=0xA5)
    T = w.torch
    x, _ = w.rows(80)
    snapshot = lambda: [t.clone() for t in (w.cache.k_codes, w.cache.v_codes, w.cache.k_scales, w.cache.v_scales)]
    a = snapshot()
    for table in (np.full((2, 2), -1), np.full((2, 2), w.pages), np.full((2, 2), 2 ** 31 - 1)):
        b = KV.KVBatch(w.i32([0, 40, 80]), w.i32([40, 40]), w.i32(table), 80, 40, 40)
        w.cache.append(x[:, 2:4], x[:, 4:], b)
        out = w.cache.attention(x[:, :2], b)
        assert bool((out == 0).all())
        for g in w.cache.gather(KV.KVRows(w.i32([0, 0]), w.i32([0, 40, 80]), w.i32(table), 80)):
            assert bool((g == 0).all())
    for lens in ([0, 0], [-5, -7]):
        b = KV.KVBatch(w.i32([0, 40, 80]), w.i32(lens), w.i32(w.table), 80, 40, 40)
        w.cache.append(x[:, 2:4], x[:, 4:], b)
        assert bool((w.cache.attention(x[:, :2], b) == 0).all())
    T.cuda.synchronize()
    assert all(T.equal(p, q) for p, q in zip(a, snapshot()))
    # token counts that do not ascend, or pass the input: clamped
    for cu in ([0, 60, 20], [5, 200, 90], [-9, -3, 400], [80, 80, 80]):
        b = KV.KVBatch(w.i32(cu), w.i32([40, 64]), w.i32(w.table), 80, 80, 64)
        w.cache.append(x[:, 2:4], x[:, 4:], b)
        w.cache.attention(x[:, :2], b)
        w.cache.attention(x[:, :2], KV.KVBatch(b.cu_new, b.kv_len, b.block_table, 80, 16, 64))
        w.cache.gather(KV.KVRows(w.i32([7, 31]), b.cu_new, b.block_table, 80))
    T.cuda.synchronize()


def test_more_new_tokens_than_length_have_no_place(torch, KV):
    w = World(torch, KV, 1, 64, 32, [64], 7)
    x, xn = w.rows(40)
    b = KV.KVBatch(w.i32([0, 40]), w.i32([33]), w.i32(w.table), 40, 40, 40)      # the first seven have position -7 .. -1
    w.cache.append(x[:, 1:2], x[:, 2:], b)
    w.oracle.append(0, 0, xn[7:, 1:2], xn[7:, 2:])
    w.held[0] = 33
    w.check_cache()
    for q in (x, x[:, :1].expand(40, 4, 64).contiguous()):      # 40 rows, 160 rows
        out = w.cache.attention(q[:, :q.shape[1] if q.shape[1] == 4 else 1], b)
        assert bool((out[:7] == 0).all()) and bool((out[7:] != 0).any(-1).all())


@pytest.mark.parametrize("dim,page,lens,first", [(64, 32, [1, 33, 200, 0, 64], [0, 5, 31, 0, 63]), (128, 64, [77, 128], [32, 0]), (256, 256, [300], [257])])
def test_gather_reads_back_what_the_codes_stand_for(torch, KV, dim, page, lens, first):
    w = World(torch, KV, 3, dim, page, lens, 8, dims=dim)
    w.append(lens)
    cu = np.concatenate([[0], np.cumsum([n - f for n, f in zip(lens, first)])])
    rows = KV.KVRows(w.i32(first), w.i32(cu), w.i32(w.table), int(cu[-1]))
    guard = [torch.full((int(cu[-1]) + 8, 3, dim), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    got = w.cache.gather(rows, out=[g[4:-4] for g in guard])
    for g in guard:
        assert bool((g[:4] == 9).all()) and bool((g[-4:] == 9).all())
    for b in range(len(lens)):
        for g, want in zip(got, w.oracle.rows(b, first[b], lens[b]) if lens[b] else (np.zeros((0, 3, dim)),) * 2):
            assert np.array_equal(g[cu[b]:cu[b + 1]].double().cpu().numpy(), want)
    # one of the two alone
    only = torch.zeros_like(got[1])
    S._check(S.lib().svdq_kv_gather(w.cache.cdesc, rows.first_token.data_ptr(), rows.cu_rows.data_ptr(), rows.block_table.data_ptr(), rows.sequences,
                                    rows.block_table.shape[1], rows.rows, None, only.data_ptr(), None), "svdq_kv_gather")
    torch.cuda.synchronize()
    assert torch.equal(only, got[1])


# ---- attention -----------------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,heads,group,page,held,new,causal,window", [
    # single tokens: contexts of one token, around the blocks and the tiles, of none before
    (128, 2, 4, 64, [0, 1, 30, 31, 32, 62, 63, 64, 127, 128, 300], [1] * 11, True, 0),
    (64, 3, 1, 32, [0, 5, 95, 700], [1] * 4, True, 0),
    (256, 1, 8, 128, [0, 33, 400], [1] * 3, True, 0),
    (128, 1, 16, 32, [500], [1], True, 0),
    (128, 1, 17, 32, [500, 3], [1, 1], True, 0),            # two tiles of sixteen rows
    (64, 2, 3, 64, [40, 0, 200, 31], [4, 3, 0, 2], True, 0),       # a few tokens, one sequence without
    (64, 2, 3, 64, [40, 0, 200, 31], [4, 3, 1, 2], True, 5),       # window inside the step
    (128, 1, 4, 64, [700, 90], [3, 1], True, 64),
    (128, 2, 2, 64, [900], [2], False, 0),                  # every key, also those behind the row
    # chunks
    (128, 2, 2, 64, [0, 37], [100, 65], True, 0),
    (64, 1, 5, 32, [0, 0, 64, 1], [33, 1, 0, 90], True, 0),
    (64, 2, 1, 128, [200], [150], True, 37),
    (64, 1, 1, 64, [100], [40], True, 1),
    (256, 1, 2, 32, [10], [70], True, 0),
    (128, 1, 3, 256, [0, 5], [129, 44], False, 0),
    (64, 1, 40, 64, [64, 0], [1, 3], True, 0),              # many heads on one
])
def test_attention_over_ragged_batches(torch, KV, dim, heads, group, page, held, new, causal, window):
    w = World(torch, KV, heads, dim, page, [h + n for h, n in zip(held, new)], dim + heads + group + len(held), q_heads=heads * group, dims=dim // 2, interleaved=group % 2 == 1)
    if any(held):
        w.append(held)
    x, xn, _, before = w.append(new, scale=1.5)
    w.attend(x, xn, new, before, causal, window)


@pytest.mark.parametrize("dim,new", [(128, 1), (128, 90), (64, 2), (64, 40)])
def test_attention_where_scales_and_scores_spread(torch, KV, dim, new):
    """Blocks of very different scales in either order, scores up to some hundred, a scale of the caller's own."""
    w = World(torch, KV, 1, dim, 64, [600 + new], 40 + dim + new, q_heads=2)
    for i, s in enumerate([1e-3, 200.0, 1e-6, 1.0, 3e4, 1e-2]):
        w.append([97], scale=s)
    x, xn, _, before = w.append([new])
    w.attend(x, xn, [new], before, scale=2e-4)
    w.attend(x, xn, [new], before, scale=3e-3)
    w.attend(x, xn, [new], before, scale=-1e-3)
    w.attend(x, xn, [new], before, scale=0.0)


def test_attention_keeps_the_small_weights_of_many_keys(torch, KV):
    """One key far above 3000 others that have e^-9 of its weight each: together they weigh a third."""
    w = World(torch, KV, 1, 64, 64, [3008], 51, gain=0.0)

    def poke(x):
        x[:, 2] = torch.arange(64, device=DEV, dtype=torch.float32) % 7 - 2.0
        x[5, 1] = 1.0
        x[5, 2] = -1.0
        x[-1, 0] = 9.0 / 8.0
    x, xn, _, before = w.append([3008], poke=poke)
    before = [3007]
    w.held = [3008]
    w.attend(x[-1:], xn[-1:], [1], before)


@pytest.mark.parametrize("new", [1, 70])
def test_attention_takes_any_strides(torch, KV, new):
    w = World(torch, KV, 2, 64, 64, [120 + new], 61, q_heads=6, dims=64)
    w.append([120])
    x, xn, _, before = w.append([new])
    by_head = torch.empty(6, new + 3, 72, dtype=torch.bfloat16, device=DEV)      # head-major, padded rows
    view = by_head[:, 1:new + 1, :64].permute(1, 0, 2)
    view.copy_(x[:, :6])
    batch, _ = w.batch([new])
    batch = KV.KVBatch(batch.cu_new, w.i32(w.held), batch.block_table, new, new, w.held[0])
    assert torch.equal(w.cache.attention(view, batch, w.rope), w.cache.attention(x[:, :6], batch, w.rope))
    again = KV.KVCache(w.pages, 2, 64, 64)
    kv = torch.empty(4, new + 3, 80, dtype=torch.bfloat16, device=DEV)
    kk, vv = kv[:2, 2:new + 2, 8:72].permute(1, 0, 2), kv[2:, 2:new + 2, 8:72].permute(1, 0, 2)
    kk.copy_(x[:, 6:8])
    vv.copy_(x[:, 8:])
    one = KV.KVBatch(batch.cu_new, w.i32([new]), batch.block_table, new, new, new)
    again.append(kk, vv, one, w.rope)
    plain = KV.KVCache(w.pages, 2, 64, 64)
    plain.append(x[:, 6:8], x[:, 8:], one, w.rope)
    assert torch.equal(again.k_codes, plain.k_codes) and torch.equal(again.v_codes, plain.v_codes) and torch.equal(again.v_scales, plain.v_scales)


@pytest.mark.parametrize("dim,heads,group,held,new", [(128, 1, 4, 5000, 1), (64, 2, 8, 3000, 3), (128, 2, 1, 300, 200), (256, 1, 2, 2500, 1)])
def test_attention_is_the_same_every_time_and_stays_inside_its_buffers(torch, KV, dim, heads, group, held, new):
    w = World(torch, KV, heads, dim, 64, [held + new] * 2, 71, q_heads=heads * group)
    batch0, _ = w.batch([held, held])
    x, _ = w.rows(2 * held)
    Q = heads * group
    w.cache.append(x[:, Q:Q + heads], x[:, Q + heads:], batch0)
    w.held = [held, held]
    batch, _ = w.batch([new, new])
    y, _ = w.rows(2 * new)
    w.cache.append(y[:, Q:Q + heads], y[:, Q + heads:], batch)
    n = w.cache.attention_workspace(batch, Q).numel()
    results = []
    for fill in (0, 0xFF, 0x5A):
        big = torch.full((n + 512,), fill, dtype=torch.uint8, device=DEV)
        ws = big[256:256 + n]
        out = torch.full((2 * new + 4, Q, dim), 3.0, dtype=torch.bfloat16, device=DEV)
        for _ in range(2):      # the second call on what the first one left
            w.cache.attention(y[:, :Q], batch, out=out[2:-2], workspace=ws)
            torch.cuda.synchronize()
            results.append(out[2:-2].clone())
            assert bool((out[:2] == 3).all()) and bool((out[-2:] == 3).all())
            assert bool((big[:256] == fill).all()) and bool((big[256 + n:] == fill).all())
    assert all(torch.equal(results[0], r) for r in results)


def test_lengths_past_the_batch_s_bound_are_still_right(torch, KV):
    w = World(torch, KV, 1, 64, 64, [900], 81, q_heads=2)
    w.append([899])
    x, xn, _, before = w.append([1])
    batch = KV.KVBatch(w.i32([0, 1]), w.i32([900]), w.i32(w.table), 1, 1, 900)
    low = KV.KVBatch(w.i32([0, 1]), w.i32([900]), w.i32(w.table), 1, 1, 300)
    a, b = w.cache.attention(x[:, :2], batch).float(), w.cache.attention(x[:, :2], low).float()
    assert float((a - b).abs().max()) <= 2.0 ** -7 * float(a.abs().max())      # (other chunks: two roundings of an output apart at most)


def test_caches_past_four_gibibytes(torch, KV):
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (heads * dim * page) + 40
    cache = KV.KVCache(pages, heads, dim, page)
    small = KV.KVCache(4, heads, dim, page)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.randn(200, 3 * heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    out = []
    for c, table in ((cache, [[pages - 1, 3, pages - 30, pages - 2]]), (small, [[0, 1, 2, 3]])):
        for first, n in ((0, 200), (200, 1)):
            b = KV.KVBatch(i32([0, n]), i32([first + n]), i32(table), n, n, 201)
            y = x[:n] if n > 1 else x[:1] * 2
            c.append(y[:, heads:2 * heads], y[:, 2 * heads:], b)
            out.append(c.attention(y[:, :heads], b))
        out += c.gather(KV.KVRows(i32([0]), i32([0, 201]), i32(table), 201))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out[:4], out[4:]))


def test_calls_follow_the_stream_and_a_graph_replays_them(torch, KV):
    w = World(torch, KV, 2, 128, 64, [2000, 700], 91, q_heads=8, dims=128)
    x, _ = w.rows(2400)
    batch0 = KV.KVBatch(w.i32([0, 1800, 2400]), w.i32([1800, 600]), w.i32(w.table), 2400, 1800, 1800)
    w.cache.append(x[:, 8:10], x[:, 10:], batch0, w.rope)
    y, _ = w.rows(2)
    batch = KV.KVBatch(w.i32([0, 1, 2]), w.i32([1801, 601]), w.i32(w.table), 2, 1, 2000)
    ws = w.cache.attention_workspace(batch, 8)
    want = []
    for i in range(3):
        z = y * (i + 1)
        w.cache.append(z[:, 8:10], z[:, 10:], batch, w.rope)
        want.append(w.cache.attention(z[:, :8], batch, w.rope, workspace=ws).clone())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step, out = torch.empty_like(y), torch.empty_like(want[0])
    with torch.cuda.stream(side):
        step.copy_(y)
        w.cache.append(step[:, 8:10], step[:, 10:], batch, w.rope)
        w.cache.attention(step[:, :8], batch, w.rope, out=out, workspace=ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        w.cache.append(step[:, 8:10], step[:, 10:], batch, w.rope)
        w.cache.attention(step[:, :8], batch, w.rope, out=out, workspace=ws)
    scales = [w.cache.k_scales.clone(), w.cache.v_scales.clone()]
    for i in (0, 1, 2, 1, 0):
        # (a block keeps the largest scale that it has had; the steps of the eager calls ended with the largest)
        step.copy_(y * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager = torch.empty_like(out)
        z = y * (i + 1)
        w.cache.append(z[:, 8:10], z[:, 10:], batch, w.rope)
        w.cache.attention(z[:, :8], batch, w.rope, out=eager, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
    assert torch.equal(out, eager) and all(torch.equal(a, b) for a, b in zip(scales, [w.cache.k_scales, w.cache.v_scales]))


def test_binding_refuses_what_the_kernels_do_not_take(torch, KV):
    w = World(torch, KV, 2, 64, 32, [64], 95)
    x, _ = w.rows(4)
    batch, _ = w.batch([4])
    for bad in (x[:, 2:4].float(), x[:, 2:3], x[:3, 2:4], x[:, 2:4].cpu(), x[:, 2:4].transpose(1, 2)):
        with pytest.raises(AssertionError):
            w.cache.append(bad, x[:, 4:], batch)
    with pytest.raises(AssertionError):
        w.cache.attention(x[:, :2], batch, out=torch.empty(4, 2, 64, device=DEV))
    with pytest.raises(S.SvdqError):
        w.cache.attention(x[:, :3], batch)      # three query heads on two
    with pytest.raises(S.SvdqError):
        w.cache.attention(x[:, :2], batch, window=-1)
    with pytest.raises(S.SvdqError):
        KV.KVCache(4, 2, 96, 64)
    odd = torch.empty(4 * 6 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(4, 6, 64)
    with pytest.raises(S.SvdqError):
        w.cache.append(odd[:, 2:4], odd[:, 4:], batch)
