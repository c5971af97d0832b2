"""Streams on the paged 8-bit cache: keys and queries normalised on the way, windows with first tokens that stay visible.  Codes and outputs are held to the definition in 64
bits within what the roundings allow (oracle/kv_stream_oracle.py derives that), over head sizes, orders of the rotation, weights, masks and cuts of the keys."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import kv_stream_oracle as W
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


class Norm:
    """Weights on the GPU and in numpy."""

    def __init__(self, torch, KV, rng, q_heads, heads, dim, per_head=False, first=0, eps=1e-6, ones=False):
        make = lambda n: None if ones else (0.3 + rng.random((n, dim) if per_head else dim) * 1.5).astype(np.float32)
        self.q, self.k, self.q_first, self.k_first, self.first, self.eps = make(q_heads), make(heads), make(q_heads), make(heads), first, np.float32(eps)
        up = lambda w: None if w is None else torch.from_numpy(w).to(DEV)
        self.dev = KV.KVNorm(up(self.q), up(self.k), eps, q_first=up(self.q_first), k_first=up(self.k_first), first_tokens=first)

    def ready(self, x, positions, side, table, interleaved):
        """x [n, heads, D] normalised and rotated, and the size of the terms"""
        x = x.astype(np.float64)
        a, b = (W.normalise(x, w, float(self.eps)) for w in (getattr(self, side), getattr(self, side + "_first")))
        return W.turn(np.where((positions < self.first)[:, None, None], b, a), positions, table, interleaved)


class Stream:
    """Sequences with a cache on the GPU; what went in is kept beside it."""

    def __init__(self, torch, KV, heads, dim, page, capacity, seed, q_heads=None, dims=None, interleaved=False, norm=None, positions=None):
        self.torch, self.KV, self.rng = torch, KV, np.random.default_rng(seed)
        self.heads, self.dim, self.page, self.q_heads, self.interleaved = heads, dim, page, q_heads or heads, interleaved
        B, self.width = len(capacity), max(1, max((c + page - 1) // page for c in capacity))
        self.pages = B * self.width + 3
        self.table = self.rng.permutation(self.pages)[:B * self.width].reshape(B, self.width).astype(np.int32)
        self.cache = KV.KVCache(self.pages, heads, dim, page)
        for t in self.buffers():
            t.fill_(0xFF)
        self.held = np.zeros(B, np.int64)
        self.rope_np, self.rope = None, None
        if dims:
            n = positions or max(capacity) + 1
            a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(dims // 2) * 2.0 / dims)
            self.rope_np = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
            self.rope = KV.Rope(torch.from_numpy(self.rope_np).to(DEV), interleaved)
        self.norm = Norm(torch, KV, self.rng, self.q_heads, heads, dim, **norm) if norm is not None else None

    def buffers(self):
        return self.cache.k_codes, self.cache.k_scales, self.cache.v_codes, self.cache.v_scales

    def batch(self, new, table=None):
        cu = np.concatenate([[0], np.cumsum(new)])
        return self.KV.KVBatch(i32(self.torch, cu), i32(self.torch, self.held), i32(self.torch, self.table if table is None else table), int(cu[-1]), int(max(new)), int(self.held.max())), cu

    def append(self, new, scale=1.0, poke=None):
        """qkv rows of the new tokens, on the GPU and in fp32"""
        T = int(np.sum(new))
        x = self.torch.from_numpy(self.rng.standard_normal((T, self.q_heads + 2 * self.heads, self.dim)) * scale).to(DEV).to(self.torch.bfloat16)
        if poke is not None:
            poke(x)
        self.held = self.held + np.asarray(new)
        batch, cu = self.batch(new)
        H, Q = self.heads, self.q_heads
        self.cache.append(x[:, Q:Q + H], x[:, Q + H:], batch, self.rope, norm=self.norm.dev if self.norm else None)
        self.torch.cuda.synchronize()
        return x, x.float().cpu().numpy(), cu

    def rows(self, b, table=None):
        """keys and values fp64 [held, heads, D] of sequence b as its bytes say, and the bytes [held, heads] of both"""
        kc, ks, vc, vs = (t.cpu().numpy() for t in self.buffers())
        k, v, kb, vb = [], [], [], []
        for blk in range((self.held[b] + 31) // 32):
            page, at = (self.table if table is None else table)[b, blk * 32 // self.page], blk * 32 % self.page // 32
            pair = [K.block_numbers(kc[page, h, at], vc[page, h, at]) for h in range(self.heads)]
            kb.append(np.tile(ks[page, :, at].astype(np.int64), (32, 1)))
            vb.append(np.tile(vs[page, :, at].astype(np.int64), (32, 1)))
            k.append(np.stack([p[0] for p in pair], 1) * np.exp2(kb[-1] - 127.0)[..., None])
            v.append(np.stack([p[1] for p in pair], 1) * np.exp2(vb[-1] - 127.0)[..., None])
        n = self.held[b]
        return tuple(np.concatenate(z)[:n] for z in (k, v, kb, vb))

    def attend(self, x, xn, new, causal=True, window=0, sinks=0, scale=None, table=None, hidden=(), **kw):
        """hidden: (sequence, first, last) tokens whose pages the table does not name"""
        batch, cu = self.batch(new, table)
        out = self.torch.full((int(cu[-1]), self.q_heads, self.dim), 7.0, dtype=self.torch.bfloat16, device=DEV)
        got = self.cache.attention(x[:, :self.q_heads], batch, self.rope, scale=scale, causal=causal, window=window, out=out, sinks=sinks,
                                   norm=self.norm.dev if self.norm else None, **kw)
        self.torch.cuda.synchronize()
        got = got.float().cpu().numpy().astype(np.float64)
        for b, n in enumerate(new):
            if n == 0:
                continue
            k, v, _, _ = self.rows(b)
            at = self.held[b] - n + np.arange(n)
            keys = np.arange(self.held[b])
            for s, lo, hi in hidden:
                if s == b:
                    keep = (keys < lo) | (keys >= hi)
                    keys, k, v = keys[keep], k[keep], v[keep]
            q = xn[cu[b]:cu[b + 1], :self.q_heads]
            q, size = self.norm.ready(q, at, "q", self.rope_np, self.interleaved) if self.norm else W.turn(q.astype(np.float64), at, self.rope_np, self.interleaved)
            want, tol = W.attention(q, size, k, v, at, keys, self.dim ** -0.5 if scale is None else scale, causal, window, sinks)
            g = got[cu[b]:cu[b + 1]]
            assert np.array_equal(np.isnan(g), np.isnan(want)), b
            ok = ~np.isnan(want)
            off = (np.abs(g - want) - tol)[ok]
            assert off.size == 0 or off.max() <= 0, (b, off.max(), np.unravel_index(np.argmax(np.where(ok, np.abs(g - want) - tol, -1)), g.shape))
        return got


# ---- norms -----------------------------------------------------------------------------------------------------------------------------------


def check_keys(w, sent):
    """sent: per sequence fp32 keys and values [held, heads, D] as they went in, and which tokens came with the last append"""
    for b, (kx, vx, last) in enumerate(sent):
        if not len(kx):
            continue
        k, v, kb, vb = w.rows(b)
        at = np.arange(len(kx))
        y, size = w.norm.ready(kx, at, "k", w.rope_np, w.interleaved)
        bad = ~(np.isfinite(y).all(-1) & np.isfinite(vx).all(-1))
        assert np.array_equal(np.isnan(k).all(-1), bad) and np.array_equal(np.isnan(k).any(-1), bad) and (v[bad] == 0).all()
        y, size, vx = np.where(bad[..., None], 0, y), np.where(bad[..., None], 0, size), np.where(bad[..., None], 0, vx).astype(np.float64)
        s = np.exp2(np.maximum(kb, 1) - 127.0)[..., None]
        tol = W.code_bounds(y, W.READY * size, kb[..., None]) + np.where(last[:, None, None], 0.0, 2.0 ** -10 * s)      # (those before were rounded again where the scale grew)
        assert (np.abs(np.where(bad[..., None], 0, k) - y) <= tol).all(), b
        s = np.exp2(np.maximum(vb, 1) - 127.0)[..., None]
        assert (np.abs(v - vx) <= W.code_bounds(vx, 0.0, vb[..., None]) + np.where(last[:, None, None], 0.0, 2.0 ** -10 * s)).all(), b
        for blk in range((len(kx) + 31) // 32):
            part = slice(32 * blk, 32 * blk + 32)
            for h in range(w.heads):
                top = np.abs(y[part, h]).max()
                assert kb[32 * blk, h] in W.scale_bytes(top, W.READY * size[part, h].max()), (b, blk, h)
                assert vb[32 * blk, h] == K.scale_byte(np.abs(vx[part, h]).max()), (b, blk, h)


@pytest.mark.parametrize("dim,heads,page,dims,inter,norm,steps", [
    (128, 2, 64, 128, False, {}, [[70, 1, 33, 0]] + [[1, 1, 1, 1]] * 3),
    (128, 5, 32, 64, True, dict(per_head=True, first=40), [[31, 32, 1], [2, 33, 0], [0, 1, 64]]),
    (128, 1, 64, 0, False, dict(first=7), [[33, 5], [1, 60]]),
    (64, 5, 128, 64, False, dict(per_head=True), [[129, 5], [1, 27], [1, 1]]),
    (64, 1, 64, 32, True, dict(ones=True, first=3), [[1], [1], [30], [1], [40]]),
    (64, 12, 32, 32, False, dict(first=1000), [[100, 3], [9, 64]]),
    (256, 2, 64, 256, False, dict(per_head=True, first=33), [[40, 3], [1, 62]]),
    (256, 1, 1024, 96, True, dict(eps=1e-2), [[37], [1]]),
    (128, 8, 64, 128, True, dict(first=512), [[700, 600]]),
])
def test_append_normalises_before_it_rotates(torch, KV, dim, heads, page, dims, inter, norm, steps):
    w = Stream(torch, KV, heads, dim, page, np.sum(steps, axis=0), 10 + dim + heads, q_heads=heads, dims=dims, interleaved=inter, norm=norm)
    sent = [[np.zeros((0, heads, dim), np.float32)] * 2 for _ in steps[0]]
    for i, new in enumerate(steps):      # (the scale of a row is divided out, but for eps and values)
        _, xn, cu = w.append(new, scale=[1.0, 3.7, 0.02, 40.0, 1e-3][i % 5])
        for b in range(len(new)):
            part = xn[cu[b]:cu[b + 1]]
            sent[b] = [np.concatenate([s, z]) for s, z in zip(sent[b], (part[:, heads:2 * heads], part[:, 2 * heads:]))]
        check_keys(w, [(k, v, np.arange(len(k)) >= len(k) - new[b]) for b, (k, v) in enumerate(sent)])
    used = {int(p) for b, n in enumerate(w.held) for p in w.table[b, :(n + page - 1) // page]}
    for p in set(range(w.pages)) - used:
        assert all((t[p].cpu().numpy() == 0xFF).all() for t in w.buffers()), "a page of no sequence was written"


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_norms_at_the_ends_of_the_range(torch, KV, dim):
    """Rows whose squares leave fp32, rows far below eps, of zeros, with numbers that are not finite: in keys, and in queries of few and of many rows."""
    w = Stream(torch, KV, 2, dim, 64, [220], 77, q_heads=4, dims=dim, norm=dict(first=5))

    def poke(x):
        x[3] *= 1e30                    # (values too)
        x[4, :6] = 3e38
        x[5, :6] *= 1e-25
        x[6, :6] = 0.0
        x[7, 4, 11] = float("nan")
        x[8, 5, 0] = float("inf")
        x[9, :6, 1:] = 0.0
        x[10, 6, 2] = -float("inf")     # a value
    x, xn, cu = w.append([200], poke=poke)
    check_keys(w, [(xn[:, 4:6], xn[:, 6:], np.ones(200, bool))])
    few = [3, 4, 5, 6, 9]
    for rows in (few, few * 12):        # (the queries of the rows above, at the last positions)
        q = torch.zeros_like(x[:len(rows)])
        q[:, :4] = x[rows, :4]
        w.held = np.array([200])
        w.attend(q, q.float().cpu().numpy(), [len(rows)], window=64, sinks=1)
    q[0, 1, 3], q[-1, 2, 7] = float("nan"), -float("inf")
    got = w.attend(q, q.float().cpu().numpy(), [len(rows)], window=64, sinks=1)
    assert np.isnan(got[0, 1]).all() and np.isnan(got[-1, 2]).all() and np.isnan(got).any((-1,)).sum() == 2
    got = w.attend(q[:3], q[:3].float().cpu().numpy(), [3], window=64)
    assert np.isnan(got[0, 1]).all() and np.isnan(got).any((-1,)).sum() == 1


@pytest.mark.parametrize("dim,heads,group,dims,inter,norm,held,new", [
    (128, 2, 4, 128, False, {}, [0, 1, 31, 32, 300], [1] * 5),
    (128, 2, 3, 64, True, dict(per_head=True, first=33), [0, 31, 300], [2, 3, 1]),
    (64, 3, 1, 64, False, dict(first=2), [0, 5, 95], [3, 1, 0]),
    (64, 1, 5, 0, False, dict(per_head=True), [40], [3]),
    (256, 1, 8, 256, True, dict(first=400), [0, 33, 400], [1] * 3),
    (256, 1, 2, 96, False, dict(per_head=True), [10, 60], [2, 7]),
    (128, 1, 17, 128, False, dict(ones=True), [500, 3], [1, 1]),
    # many rows
    (128, 2, 2, 128, True, dict(first=64), [0, 37], [200, 165]),
    (64, 1, 5, 32, False, dict(per_head=True, first=70), [0, 0, 64], [133, 1, 90]),
    (256, 1, 2, 256, False, dict(per_head=True), [10], [170]),
    (64, 1, 4, 0, False, dict(), [100], [140]),
])
def test_attention_normalises_its_queries(torch, KV, dim, heads, group, dims, inter, norm, held, new):
    w = Stream(torch, KV, heads, dim, 64, [h + n for h, n in zip(held, new)], dim + heads + group, q_heads=heads * group, dims=dims, interleaved=inter, norm=norm)
    if any(held):
        w.append(held)
    x, xn, _ = w.append(new, scale=3.0)
    w.attend(x, xn, new)
    w.attend(x, xn, new, causal=False)
    w.attend(x, xn, new, window=33, sinks=5)


def test_weights_of_the_wrong_shape_are_refused(torch, KV):
    w = Stream(torch, KV, 2, 64, 32, [40], 1, q_heads=4, norm={})
    x, _, _ = w.append([10])
    batch, _ = w.batch([10])
    t = lambda *s: torch.ones(*s, device=DEV)
    for norm in (KV.KVNorm(t(32), t(32)), KV.KVNorm(t(2, 64), t(4, 64)), KV.KVNorm(q_first=t(128), k_first=t(128))):
        with pytest.raises(AssertionError):
            w.cache.append(x[:, 4:6], x[:, 6:], batch, norm=norm)
        with pytest.raises(AssertionError):
            w.cache.attention(x[:, :4], batch, norm=norm)
    for make in (lambda: KV.KVNorm(t(64), t(2, 64)), lambda: KV.KVNorm(t(64).half()), lambda: KV.KVNorm(t(128)[::2]), lambda: KV.KVNorm(t(4, 64), q_first=t(2, 64)),
                 lambda: KV.KVNorm(t(64), t(128)), lambda: KV.KVNorm(t(1, 2, 64))):
        with pytest.raises(AssertionError):
            make()


# ---- first tokens that stay visible ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dim,heads,group,page,held,new,window,sinks", [
    # single tokens: windows that begin in the first tokens, touch them, lie far behind
    (128, 2, 4, 64, [0, 3, 4, 5, 35, 36, 37, 68, 100, 300, 900], [1] * 11, 33, 4),
    (128, 1, 4, 32, [700], [1], 1, 1),
    (64, 3, 1, 32, [0, 95, 700], [1] * 3, 64, 33),
    (64, 3, 1, 128, [95, 700], [1] * 2, 40, 500),              # more first tokens than lie before the window
    (256, 1, 8, 128, [33, 400, 1000], [1] * 3, 100, 64),
    (128, 1, 4, 64, [5000], [1], 2500, 1300),                  # the keys in parts
    (64, 2, 3, 64, [40, 0, 200, 31], [4, 3, 0, 2], 5, 3),      # window inside the step
    (128, 1, 17, 32, [500, 3], [1, 1], 64, 31),
    (128, 1, 4, 64, [700], [1], 2 ** 31 - 1, 2 ** 31 - 1),
    # chunks
    (128, 2, 2, 64, [0, 37, 900], [100, 65, 200], 50, 4),
    (64, 2, 1, 128, [600], [350], 37, 65),
    (64, 1, 1, 64, [1000], [240], 1, 1),
    (256, 1, 2, 32, [510], [170], 130, 64),
    (128, 1, 4, 64, [700], [300], 200, 128),
    (128, 1, 4, 64, [700], [300], 200, 129),
    (128, 1, 4, 64, [64], [300], 64, 64),
    (128, 1, 2, 64, [3000], [300], 1500, 1000),                # in parts
    (64, 1, 40, 64, [64, 900], [1, 3], 40, 33),
    (128, 8, 4, 64, [2000] + [300 * i for i in range(8)], [300] + [1] * 8, 400, 40),      # beside single tokens
])
def test_the_first_tokens_stay_visible(torch, KV, dim, heads, group, page, held, new, window, sinks):
    w = Stream(torch, KV, heads, dim, page, [h + n for h, n in zip(held, new)], dim + heads + group + len(held) + sinks % 97, q_heads=heads * group, dims=dim // 2)
    w.append(held)
    x, xn, _ = w.append(new, scale=1.5)
    w.attend(x, xn, new, window=window, sinks=sinks)


@pytest.mark.parametrize("sequences,heads,group,held,new,window,sinks,norm", [
    (4, 8, 4, 3700, 512, 2100, 70, dict(first=100)),        # row tiles of 256 (tests/test_kv_stream_plan.py has the rule)
    (32, 8, 1, 3900, 256, 0, 0, dict(per_head=True)),
    (32, 4, 2, 3968, 130, 4096, 1, None),
])
def test_the_larger_tiles(torch, KV, sequences, heads, group, held, new, window, sinks, norm):
    w = Stream(torch, KV, heads, 128, 128, [held + new] * sequences, 70 + sequences, q_heads=heads * group, dims=128, norm=norm)
    w.append([held] * sequences)
    x, xn, _ = w.append([new] * sequences)
    got = w.attend(x[:new], xn[:new], [new] + [0] * (sequences - 1), window=window, sinks=sinks)      # alone: row tiles of 128
    batch, cu = w.batch([new] * sequences)
    out = w.cache.attention(x[:, :heads * group], batch, w.rope, window=window, sinks=sinks, norm=w.norm.dev if norm is not None else None).float().cpu().numpy()
    assert np.abs(out[:new] - got).max() <= 2.0 ** -7 * np.abs(got).max()
    for b in (1, sequences - 1):
        at, part = held + np.arange(new), slice(cu[b], cu[b + 1])
        k, v, _, _ = w.rows(b)
        some = np.unique(np.concatenate([np.arange(0, new, 37), [new - 1]]))      # (rows of all wavefronts)
        q = xn[part, :heads * group][some]
        q, size = w.norm.ready(q, at[some], "q", w.rope_np, False) if norm is not None else W.turn(q.astype(np.float64), at[some], w.rope_np, False)
        want, tol = W.attention(q, size, k, v, at[some], np.arange(held + new), 128 ** -0.5, True, window, sinks)
        assert (np.abs(out[part][some] - want) <= tol).all(), b


@pytest.mark.parametrize("dim,new,group", [(128, 1, 4), (128, 90, 4), (64, 2, 2), (64, 200, 1), (256, 1, 1), (256, 90, 2)])
def test_first_tokens_of_other_scales(torch, KV, dim, new, group):
    """Blocks of very different scales: those of the first tokens and of the window meet a block at a time, and what no row sees leaves no trace."""
    w = Stream(torch, KV, 1, dim, 64, [900 + new], 40 + dim + new, q_heads=group)
    for s in (1e-3, 200.0, 1e30, 1e-6, 1.0, 3e4, 1e-2):
        w.append([128], scale=s)
    x, xn, _ = w.append([new])
    w.attend(x, xn, [new], scale=1e-4, window=300, sinks=70)
    w.attend(x, xn, [new], scale=3e-3, window=40, sinks=3)


@pytest.mark.parametrize("dim,new,group,window,sinks", [(128, 1, 4, 100, 10), (64, 3, 2, 200, 64), (128, 260, 2, 100, 10), (256, 200, 1, 65, 40), (64, 300, 1, 130, 100)])
def test_pages_between_are_not_read(torch, KV, dim, new, group, window, sinks):
    """What lies between the first tokens and the windows may be given back, or hold anything: the same bits.  Without first tokens the call is the one without the argument."""
    w = Stream(torch, KV, 2, dim, 32, [1500], 5, q_heads=2 * group, dims=dim)
    w.append([1500 - new])
    x, xn, _ = w.append([new])
    batch, _ = w.batch([new])
    q = x[:, :2 * group]
    plain = w.cache.attention(q, batch, w.rope, window=window)
    assert torch.equal(plain, w.cache.attention(q, batch, w.rope, window=window, sinks=0))
    assert torch.equal(w.cache.attention(q, batch, w.rope, causal=False), w.cache.attention(q, batch, w.rope, causal=False, window=window, sinks=sinks))
    assert torch.equal(w.cache.attention(q, batch, w.rope, sinks=sinks), w.cache.attention(q, batch, w.rope))
    want = w.attend(x, xn, [new], window=window, sinks=sinks)
    lo, hi = (sinks + 31) // 32, (1500 - new + 1 - window) // 32      # pages wholly between
    table = w.table.copy()
    table[0, lo:hi] = [-1, w.pages, 2 ** 31 - 1][new % 3]
    assert np.array_equal(w.attend(x, xn, [new], window=window, sinks=sinks, table=table), want)
    for t in w.buffers():
        t[torch.from_numpy(w.table[0, lo:hi].astype(np.int64)).to(DEV)] = 0xFF
    assert np.array_equal(w.attend(x, xn, [new], window=window, sinks=sinks), want)
    # pages of the first tokens that are gone: those are not seen
    table[0, 0] = -1
    w.attend(x, xn, [new], window=window, sinks=sinks, table=table, hidden=[(0, 0, 32)])


def test_tokens_without_a_position_see_no_first_tokens(torch, KV):
    w = Stream(torch, KV, 1, 64, 32, [64], 7, q_heads=2)
    w.append([33])
    for n in (40, 200):
        q = torch.randn(n, 2, 64, device=DEV).to(torch.bfloat16)
        b = KV.KVBatch(i32(torch, [0, n]), i32(torch, [33]), i32(torch, w.table), n, n, 33)
        out = w.cache.attention(q, b, window=8, sinks=4)
        assert bool((out[:n - 33] == 0).all()) and bool((out[n - 33:] != 0).any(-1).all())


def test_a_stream_in_a_captured_step(torch, KV):
    """Append and attention of one token each, lengths counted up by the graph: every replay as the eager call."""
    B, H, G, D, P = 3, 2, 4, 128, 64
    make = lambda: Stream(torch, KV, H, D, P, [400, 200, 300], 9, q_heads=H * G, dims=D, norm=dict(first=10))
    eager, graphed = make(), make()
    for w in (eager, graphed):
        w.append([150, 3, 60])
    steps = torch.randn(12, B, (G + 2) * H, D, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV).to(torch.bfloat16)

    def step(w, x, batch, out, ws):
        w.cache.append(x[:, H * G:H * G + H], x[:, H * G + H:], batch, w.rope, norm=w.norm.dev)
        w.cache.attention(x[:, :H * G], batch, w.rope, window=70, sinks=5, norm=w.norm.dev, out=out, workspace=ws)

    def parts(w):
        length, x = i32(torch, w.held), torch.zeros_like(steps[0])
        batch = KV.KVBatch(i32(torch, range(B + 1)), length, i32(torch, w.table), B, 1, 400)
        return length, x, batch, torch.empty(B, H * G, D, dtype=torch.bfloat16, device=DEV), w.cache.attention_workspace(batch, H * G)
    length, x, batch, out, ws = parts(graphed)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(graphed, x, KV.KVBatch(batch.cu_new, i32(torch, [0] * B), batch.block_table, B, 1, 400), out, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        length.add_(1)
        step(graphed, x, batch, out, ws)
    e_length, e_x, e_batch, e_out, e_ws = parts(eager)
    for i in range(12):
        x.copy_(steps[i])
        graph.replay()
        e_x.copy_(steps[i])
        e_length.add_(1)
        step(eager, e_x, e_batch, e_out, e_ws)
        torch.cuda.synchronize()
        assert torch.equal(out, e_out), i
    assert all(torch.equal(a, b) for a, b in zip(eager.buffers(), graphed.buffers()))
