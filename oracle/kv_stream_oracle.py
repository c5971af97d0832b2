"""Oracle of what streams and branches do with the paged 8-bit cache of keys and values: norms of heads, windows with first tokens that stay visible, compaction of
tokens, pages that are shared.  Plain numpy in 64 bits.  Test infrastructure.
"""
from __future__ import annotations

import numpy as np

from oracle import kv_oracle as K


def normalise(x, weight, eps):
    """w x / sqrt(mean x^2 + eps) over the last axis; x fp64 [..., heads, D], weight None, [D] or [heads, D].  (Squares of 64-bit numbers hold those of bf16 ones.)"""
    with np.errstate(invalid="ignore", over="ignore"):
        y = x / np.sqrt(np.square(x).mean(-1, keepdims=True) + eps)
        return y if weight is None else y * np.asarray(weight, np.float64)


def turn(x, positions, table, interleaved, back=False):
    """x fp64 [n, heads, D] turned by the angles of its tokens' positions [n] or [n, heads] (back: the other way, and divided by the squared size of the table's entries).
    Returns it and, per element, |a cos| + |b sin|: what a rounding of its two products is relative to."""
    size = np.abs(x)
    if table is None:
        return x.copy(), size
    y, size = x.copy(), size.copy()
    dims = table.shape[1]
    row = np.asarray(table, np.float64)[np.minimum(positions, table.shape[0] - 1)]
    row = row[:, None] if row.ndim == 2 else row
    c, s = row[..., :dims // 2], row[..., dims // 2:]
    if back:
        c, s = c / (c * c + s * s), -s / (c * c + s * s)
    i, j = (np.arange(0, dims, 2), np.arange(1, dims, 2)) if interleaved else (np.arange(dims // 2), np.arange(dims // 2, dims))
    a, b = x[..., i], x[..., j]
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
        size[..., i], size[..., j] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return y, size


# What fp32 may make of a normalised and rotated number, relative to |a cos| + |b sin|.  Squares of up to 256 channels: each is rounded once in its fma, a lane adds up to
# 64 of them and lanes meet in up to four additions, 68 roundings of the sum at most, that is 34 of the factor; the mean, eps and the reciprocal root (1 ulp = two halves): 4;
# two products of the norm, one and a sum of the rotation: 4.  42 * 2^-24 < 2^-18.
READY = 2.0 ** -18


def code_bounds(y, slack, byte):
    """What an E4M3 code times the scale of `byte` may be off from y, which fp32 knows to `slack`: half a step of the number (2^-4 of a normal one, 2^-10 of the scale below)
    and what the slack moves, itself rounded with it."""
    s = np.exp2(np.maximum(np.asarray(byte, np.float64), 1.0) - 127)
    return np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s) + (1.0 + 2.0 ** -3) * slack


def scale_bytes(amax, slack):
    """The bytes that a maximum may get which fp32 knows to `slack`."""
    return {K.scale_byte(max(amax - slack, 0.0)), K.scale_byte(amax), K.scale_byte(amax + slack)}


def seen(positions, keys, causal, window, sinks):
    """[n, L]: which of the keys' positions each row sees"""
    p, j = np.asarray(positions)[:, None], np.asarray(keys)[None]
    if not causal:
        return np.broadcast_to(p >= 0, (p.shape[0], j.shape[1])).copy()
    ok = j <= p
    if window > 0:
        ok &= (j > p - window) | (j < sinks)
    return ok


def attention(q, size, k, v, positions, keys, scale, causal=True, window=0, sinks=0):
    """q fp64 [n, q_heads, D] (ready to be multiplied; fp32 knows it to READY * size), k, v fp64 [L, heads, D] at positions `keys`.  Returns the output and what it may be off by:
    kv_oracle.attention derives the terms for scores, weights, sums, values and the output; a score owes scale READY sum |k| size to the queries beside."""
    n, Hq, D = q.shape
    L, H, _ = k.shape
    ok = seen(positions, keys, causal, window, sinks)
    out, tol = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    some = ok.any(1)
    if not some.any():
        return out, tol
    for h in range(Hq):
        kk, vv = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
        with np.errstate(invalid="ignore", over="ignore"):
            s = np.where(ok, q[:, h] @ kk.T * scale, -np.inf)
            bad = (ok & ~np.isfinite(s)).any(1)
            p = np.exp(s - np.where(some, s.max(1), 0.0)[:, None])
            p = np.where(ok, p, 0.0) / np.where(some, np.where(ok, p, 0.0).sum(1), 1.0)[:, None]
            vz, kz = np.where(np.isfinite(vv), vv, 0.0), np.where(np.isfinite(kk), np.abs(kk), 0.0)
            out[:, h] = p @ vz
            d = abs(scale) * np.where(ok, (2.0 ** -11 + 2.0 ** -16) * (np.abs(q[:, h]) @ kz.T) + READY * (size[:, h] @ kz.T), 0.0).max(1)
            most = np.where(ok, np.abs(vz).max(1), 0.0).max(1)
            tol[:, h] = (2.0 ** -8 * np.abs(out[:, h]) + (np.expm1(2 * d) + 2.0 ** -11 + 2.0 ** -14)[:, None] * (p @ np.abs(vz))
                         + ((ok.sum(1) * 2.0 ** -33 + 2.0 ** -30) * most)[:, None])
        out[bad, h] = np.nan
    return out, tol



def moved_key(k, old, new, table, interleaved):
    """Keys fp64 [n, heads, D] turned from positions old ([n] or [n, heads]) to new [n].  Returns them and what fp32 may be off by: with u = 2^-24, cosines and sines of the
    difference come of three products and sums and a division by a reciprocal of 1 ulp (under 12 u of |c1 c0| + |s1 s0| over c0^2 + s0^2, which is at most
    the ratio g of the sizes of the two entries), the turning adds two products and a sum (3 u): (12 + 3) u g (|a| + |b|) < 2^-20 g (|a| + |b|); a code times its scale is exact."""
    back, _ = turn(k, old, table, interleaved, back=True)
    out, _ = turn(back, new, table, interleaved)
    stays = np.asarray(old) == (np.asarray(new) if np.ndim(old) == 1 else np.asarray(new)[:, None])
    stays = stays[:, None, None] if np.ndim(old) == 1 else stays[..., None]
    out = np.where(stays, k, out)
    slack = np.zeros_like(k)
    if table is not None:
        dims = table.shape[1]
        i, j = (np.arange(0, dims, 2), np.arange(1, dims, 2)) if interleaved else (np.arange(dims // 2), np.arange(dims // 2, dims))
        t = np.asarray(table, np.float64)
        size = lambda p: np.sqrt(t[np.minimum(p, len(t) - 1), :dims // 2] ** 2 + t[np.minimum(p, len(t) - 1), dims // 2:] ** 2)
        lift = lambda z: z[:, None] if z.ndim == 2 else z
        g = lift(size(np.asarray(new))) / lift(size(np.asarray(old)))
        both = 2.0 ** -20 * g * (np.abs(k[..., i]) + np.abs(k[..., j]))
        slack[..., i], slack[..., j] = both, both
    return out, np.where(stays, 0.0, slack)


class Pages:
    """Counts of pages and tables whose rows share them, one entry after another."""

    def __init__(self, pages, page_tokens):
        self.refs, self.P = [0] * pages, page_tokens

    def page(self, g):
        return 0 <= g < len(self.refs)

    def release(self, table, first=None, end=None):
        for b, row in enumerate(table):
            for e, g in enumerate(row):
                if e * self.P >= (0 if first is None else first[b]) and (end is None or (e + 1) * self.P <= end[b]):
                    if self.page(g):
                        self.refs[g] -= 1
                    row[e] = -1

    def fork(self, from_table, from_len, parent, to_table, to_len):
        for i, p in enumerate(parent):
            row, to_len[i] = to_table[i], 0
            if 0 <= p < len(from_table):
                to_len[i] = min(max(from_len[p], 0), min(len(from_table[p]), len(row)) * self.P)
            for e in range(len(row)):
                g = from_table[p][e] if e * self.P < to_len[i] else -1
                row[e] = g if self.page(g) else -1
                if self.page(g):
                    self.refs[g] += 1

    def reserve(self, table, new, lens):
        """The copies (page, to page, tokens) of every sequence, and how many entries got no page.  An entry that names no page, of a page whose first tokens are no new ones, gets
        none: nothing holds those tokens, and a page that was another's would show its.  Where all entries that name a shared page are such ones, of one place in their rows, the first
        sequence keeps it."""
        free = [g for g, n in enumerate(self.refs) if n <= 0]
        was, missing, copies, holders = list(self.refs), 0, [], {}
        lens = [min(max(n, 0), len(row) * self.P) for row, n in zip(table, lens)]
        entries = [range(max(length - n, 0) // self.P, (length + self.P - 1) // self.P) if n > 0 else () for n, length in zip(new, lens)]
        for b, row in enumerate(table):
            for e in entries[b]:
                holders.setdefault((e, row[e]), []).append(b)
        for b, (row, n, length) in enumerate(zip(table, new, lens)):
            before = max(length - n, 0)
            copy = (-1, -1, 0)
            for e in entries[b]:
                g = row[e]
                if self.page(g) and (was[g] <= 1 or len(holders[e, g]) == was[g] and b == holders[e, g][0]):
                    continue
                if not self.page(g) and e * self.P < before:
                    missing += 1
                    continue
                if self.page(g):
                    self.refs[g] -= 1
                row[e] = free.pop(0) if free else -1
                if row[e] < 0:
                    missing += 1
                    continue
                self.refs[row[e]] = 1
                if self.page(g) and e * self.P < before:
                    copy = (g, row[e], before - e * self.P)
            copies.append(copy)
        return copies, missing
