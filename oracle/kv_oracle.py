"""Oracle of the paged 8-bit cache of keys and values and of attention over it: plain numpy, one block and one row at a time.

Test infrastructure.  The quantizer's roundings are written in the fp32 operations that define them; attention is in 64 bits.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32


def e4m3_values() -> np.ndarray:
    """The number that each of the 256 codes stands for (4 exponent bits, bias 7, 3 mantissa bits; no infinities, 127 is NaN)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0 ** -9
        out[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return out


VALUES = e4m3_values()


def e4m3_round(x) -> np.ndarray:
    """The nearest E4M3 number, ties to even; |x| <= 448."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
    step = np.exp2(e - 3)
    return np.rint(x / step) * step


def scale_byte(amax) -> int:
    """Byte of the smallest power of two s >= 2^-126 with amax <= 448 s; 0 for amax = 0."""
    if amax == 0:
        return 0
    e = -126
    while float(amax) > 448.0 * 2.0 ** e:
        e += 1
    return e + 127


def rotate(x, pos, table, interleaved):
    """x fp32 [heads, D] at position pos; table fp32 [positions, dims]; every product and sum rounded to fp32."""
    x = np.array(x, np.float32)
    if table is None:
        return x
    dims = table.shape[1]
    row = table[min(pos, table.shape[0] - 1)]
    c, s = row[:dims // 2], row[dims // 2:]
    i, j = (np.arange(0, dims, 2), np.arange(1, dims, 2)) if interleaved else (np.arange(dims // 2), np.arange(dims // 2, dims))
    a, b = x[:, i].copy(), x[:, j].copy()
    with np.errstate(invalid="ignore", over="ignore"):
        x[:, i] = a * c - b * s
        x[:, j] = b * c + a * s
    return x


class Cache:
    """Sequences by number: lists of blocks with a byte per head and the numbers that their codes stand for (before the scale)."""

    def __init__(self, heads, dim):
        self.heads, self.dim = heads, dim
        self.k, self.v = {}, {}      # (sequence, block) -> [bytes [heads], numbers [heads, 32, dim]]

    def append(self, seq, held, k, v, table=None, interleaved=False):
        """held tokens are there; k, v fp32 [n, heads, dim] come behind them."""
        n = k.shape[0]
        k = np.stack([rotate(k[i], held + i, table, interleaved) for i in range(n)]) if n else k
        bad = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))           # [n, heads]
        for blk in range(held // BLOCK, (held + n + BLOCK - 1) // BLOCK):
            at = [i for i in range(n) if (held + i) // BLOCK == blk]
            fresh = held <= blk * BLOCK
            for x, store, empty in ((k, self.k, np.nan), (v, self.v, 0.0)):
                if fresh:
                    store[seq, blk] = [np.zeros(self.heads, int), np.zeros((self.heads, BLOCK, self.dim))]
                byte, num = store[seq, blk]
                for h in range(self.heads):
                    good = [i for i in at if not bad[i, h]]
                    amax = max((float(np.abs(x[i, h]).max()) for i in good), default=0.0)
                    new = max(int(byte[h]), scale_byte(amax))
                    if new > byte[h]:
                        num[h] = e4m3_round(num[h] * 2.0 ** (int(byte[h]) - new))
                    byte[h] = new
                    for i in at:
                        num[h, (held + i) % BLOCK] = empty if bad[i, h] else e4m3_round(x[i, h].astype(np.float64) * 2.0 ** (127 - max(new, 1)))

    def rows(self, seq, first, last):
        """keys and values fp64 [last - first, heads, dim]"""
        out = []
        for store in (self.k, self.v):
            r = np.empty((last - first, self.heads, self.dim))
            for t in range(first, last):
                byte, num = store[seq, t // BLOCK]
                r[t - first] = num[:, t % BLOCK] * np.exp2(byte.astype(float) - 127)[:, None]
            out.append(r)
        return out


def block_numbers(codes_k, codes_v):
    """Canonical numbers [32, D] of one block's keys and values from their bytes in the cache's order."""
    D = codes_k.size // BLOCK
    k = VALUES[codes_k.reshape(BLOCK, D)]
    v = np.empty((BLOCK, D))
    flat = codes_v.reshape(-1)
    for t in range(BLOCK):
        g, j = 2 * (t // 16) + (t % 8) // 4, 4 * ((t % 16) // 8) + t % 4
        d = np.arange(D)
        v[t] = VALUES[flat[(((d // 32 * 16 + d % 16) * 4 + g) * 2 + d % 32 // 16) * 8 + j]]
    return k, v


def attention(q, k, v, positions, scale, causal, window):
    """q fp64 [n, q_heads, D] (rotated), k, v fp64 [L, heads, D].  Returns the output and, per output, what its arithmetic may be off by:
    f16 queries (11 bits, relative error 2^-11) and fp32 sums of up to 256 products (2^-16), hence at most d = (2^-11 + 2^-16) scale sum|q k| of a score and
    e^(2 d) - 1 of a weight after normalization; f16 weights (2^-11, and half of 2^-32 of the largest below f16's normal numbers); fp32 sums and exponents
    (2^-14 of the sum of magnitudes: exponents of 100 are off by 2^-17); f16 values below its normal numbers (2^-30 of the largest); bf16 output (2^-8)."""
    n, Hq, D = q.shape
    L, H, _ = k.shape
    out, tol = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    for h in range(Hq):
        kk, vv = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
        for i in range(n):
            lo, hi = 0, L
            if causal:
                hi = max(0, min(L, positions[i] + 1))
                if window:
                    lo = max(0, positions[i] + 1 - window)
            if hi <= lo:
                continue
            s = kk[lo:hi] @ q[i, h] * scale
            if not np.isfinite(s).all():
                out[i, h] = np.nan
                continue
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ vv[lo:hi]
            d = (2.0 ** -11 + 2.0 ** -16) * abs(scale) * (np.abs(kk[lo:hi]) @ np.abs(q[i, h])).max()
            most = np.abs(vv[np.isfinite(vv).all(-1)]).max()
            tol[i, h] = 2.0 ** -8 * np.abs(out[i, h]) + (np.expm1(2 * d) + 2.0 ** -11 + 2.0 ** -14) * (p @ np.abs(vv[lo:hi])) + ((hi - lo) * 2.0 ** -33 + 2.0 ** -30) * most
    return out, tol
