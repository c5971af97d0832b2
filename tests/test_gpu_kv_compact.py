"""Compaction of the paged 8-bit cache of keys and values: every moved token against what it was, turned to its new position and rounded anew; bytes, tokens before the moves,
pages of no sequence, moves in place by way of the workspace."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S
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


def check(old, new, to_first, tokens, table, interleaved, heads, before):
    """old, new: rows() before and after of one sequence (new: its to_first + n tokens); tokens [n] or [heads, n]; before: rows() of what the new place held"""
    n = tokens.shape[-1]
    pick = lambda z: z[tokens] if tokens.ndim == 1 else np.stack([z[tokens[h], h] for h in range(heads)], 1)
    k0, v0 = pick(old[0]), pick(old[1])
    places = to_first + np.arange(n)
    k1, v1, kb, vb = (z[to_first:to_first + n] for z in new)
    want, slack = W.moved_key(np.where(np.isnan(k0), 0.0, k0), tokens if tokens.ndim == 1 else tokens.T, places, table, interleaved) if table is not None else (np.where(np.isnan(k0), 0.0, k0), 0.0 * v0)
    bad = np.isnan(k0).any(-1) | np.isnan(v0).any(-1)
    assert np.array_equal(np.isnan(k1).all(-1), bad) and np.array_equal(np.isnan(k1).any(-1), bad) and (v1[bad] == 0).all()
    z = lambda x: np.where(bad[..., None], 0.0, x)
    want, slack, v0 = z(want), z(slack), z(v0)
    assert (np.abs(z(k1) - want) <= W.code_bounds(want, slack, kb[..., None])).all()
    assert (np.abs(v1 - v0) <= W.code_bounds(v0, 0.0, vb[..., None])).all()
    # (codes at a scale that is not smaller than theirs was, and normal there, are the numbers themselves)
    exact = np.abs(v0) >= 2.0 ** -6 * np.exp2(vb - 127.0)[..., None]
    assert (np.where(exact, v1, v0) == v0).all()
    for blk in range(to_first // 32, (to_first + n + 31) // 32):
        here = (places // 32) == blk
        for h in range(heads):
            for x, sl, byte, was in ((want, slack, kb, before[2]), (v0, 0.0 * v0, vb, before[3])):
                held = int(was[blk * 32, h]) if blk * 32 < to_first else 0
                assert byte[here][0, h] in {max(held, b) for b in W.scale_bytes(np.abs(x[here, h]).max(), sl[here, h].max())}, (blk, h)
    # what was there before: its codes, or those rounded again where the scale grew
    for x, y, byte, was in ((before[0], new[0], new[2], before[2]), (before[1], new[1], new[3], before[3])):
        part = slice(to_first // 32 * 32, to_first)
        grown = np.exp2(np.maximum(byte[part], 1) - 127.0)[..., None] * (byte[part] > was[part])[..., None]
        assert (np.abs(y[part] - x[part]) <= 2.0 ** -10 * grown).all()
        assert np.array_equal(y[:part.start], x[:part.start])


@pytest.mark.parametrize("dim,heads,page,to_page,dims,inter,held,kept,to_first,per_head", [
    (128, 2, 64, 64, 128, False, [300, 70, 1, 33], [150, 70, 1, 0], [0, 0, 0, 0], False),
    (128, 3, 64, 64, 0, False, [300, 129], [100, 64], [0, 5], False),
    (128, 5, 32, 128, 64, True, [400], [64], [37], False),              # pages of another size
    (64, 2, 128, 32, 64, False, [257, 31], [256, 31], [1, 95], False),
    (64, 12, 64, 64, 32, True, [90, 300], [50, 33], [31, 64], False),
    (256, 2, 64, 64, 256, False, [100, 200], [77, 1], [0, 63], False),
    (256, 1, 1024, 1024, 96, True, [1500], [1300], [0], False),
    (128, 4, 64, 64, 128, False, [500, 64, 40], [100, 64, 7], [0, 0, 33], True),
    (64, 3, 32, 32, 0, True, [700], [40], [3], True),
    (256, 2, 64, 64, 128, False, [300], [33], [0], True),
    (128, 8, 64, 64, 128, False, [5000, 3000], [4000, 2900], [0, 40], False),      # heads in turn
])
@pytest.mark.parametrize("order", ["ascending", "any"])
def test_moved_tokens_are_what_they_were(torch, KV, dim, heads, page, to_page, dims, inter, held, kept, to_first, per_head, order):
    rng = np.random.default_rng(dim + heads + sum(kept))
    w = Stream(torch, KV, heads, dim, page, held, 3 + dim, dims=dims, interleaved=inter, positions=max(held) + max(to_first) + 1)
    at = np.zeros(len(held), int)
    for i in range(4):      # (blocks of different scales)
        part = [h // 4 if i < 3 else h - 3 * (h // 4) for h in held]
        if sum(part):
            w.append(part, scale=[1.0, 30.0, 0.01, 2.0][i])
    new_held = [t + n for t, n in zip(to_first, kept)]
    d = Stream(torch, KV, heads, dim, to_page, new_held, 5 + dim, dims=dims, interleaved=inter, positions=max(held) + max(to_first) + 1)
    if sum(to_first):
        d.append(to_first, scale=0.5)
    cu = np.concatenate([[0], np.cumsum(kept)])
    lists = []
    for h, n in zip(held, kept):
        one = [rng.permutation(h)[:n] if order == "any" else np.sort(rng.permutation(h)[:n]) for _ in range(heads if per_head else 1)]
        lists.append(np.stack(one))
    tokens = np.concatenate(lists, 1)
    if not per_head:
        tokens = tokens[0]
    old = [w.rows(b) for b in range(len(held))]
    before = [d.rows(b) if d.held[b] else (np.zeros((0, heads, dim)),) * 2 + (np.zeros((0, heads), int),) * 2 for b in range(len(held))]
    moves = KV.KVMoves(i32(torch, cu), i32(torch, tokens), i32(torch, to_first), i32(torch, w.table), i32(torch, d.table), int(cu[-1]))
    reads = [t.clone() for t in w.buffers()]
    staged = [t.clone() for t in d.buffers()]
    d.cache.compact(moves, rope=w.rope, source=w.cache)
    torch.cuda.synchronize()
    d.held = np.asarray(new_held)
    for b in range(len(held)):
        if kept[b]:
            part = tokens[..., cu[b]:cu[b + 1]]
            check(old[b], d.rows(b), to_first[b], part, w.rope_np, inter, heads, before[b])
    assert all(torch.equal(a, b) for a, b in zip(reads, w.buffers()))
    used = {int(p) for b, n in enumerate(new_held) for p in d.table[b, :(n + to_page - 1) // to_page]}
    for p in set(range(d.pages)) - used:
        assert all((t[p] == 0xFF).all() for t in d.buffers()), "a page of no sequence was written"
    # by way of the workspace, and again: the same bytes
    direct = [t.clone() for t in d.buffers()]
    for t, s in zip(d.buffers(), staged):
        t.copy_(s)
    ws = d.cache.compact_workspace(moves)
    guard = torch.full((ws.numel() + 4096,), 0xA5, dtype=torch.uint8, device=DEV)
    for _ in range(2):
        d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=guard[:-4096])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(direct, d.buffers())) and bool((guard[-4096:] == 0xA5).all())


@pytest.mark.parametrize("dim,dims,to_first,order", [(128, 128, 0, "ascending"), (64, 32, 37, "any"), (256, 0, 5, "reversed")])
def test_a_sequence_shrinks_in_place(torch, KV, dim, dims, to_first, order):
    w = Stream(torch, KV, 2, dim, 64, [700, 130], 21 + dim, dims=dims)
    w.append([350, 65])
    w.append([350, 65], scale=9.0)
    rng = np.random.default_rng(4)
    lists = [to_first + rng.permutation(700 - to_first)[:400], to_first + rng.permutation(130 - to_first)[:60]]
    lists = [np.sort(x) if order == "ascending" else np.sort(x)[::-1] if order == "reversed" else x for x in lists]
    old = [w.rows(b) for b in range(2)]
    table = i32(torch, w.table)
    moves = KV.KVMoves(i32(torch, [0, 400, 460]), i32(torch, np.concatenate(lists)), i32(torch, [to_first] * 2), table, table, 460)
    w.cache.compact(moves, rope=w.rope, workspace=w.cache.compact_workspace(moves))
    torch.cuda.synchronize()
    w.held = np.array([to_first + 400, to_first + 60])
    for b in range(2):
        check(old[b], w.rows(b), to_first, lists[b], w.rope_np, False, 2, old[b])
    x, xn, _ = w.append([3, 1])      # and goes on
    w.attend(x, xn, [3, 1])


def test_tokens_that_keep_their_position_keep_their_numbers(torch, KV):
    """Also where the cosines and sines are scaled, and a code is the largest.  (A byte is that of the numbers that are held: 1.76 * 2^8 steps of a scale were rounded to
    1.75 * 2^8, which half the scale holds too.)"""
    w = Stream(torch, KV, 2, 128, 64, [200], 31, dims=128)

    def poke(x):
        x[:, 2:4, 5] = 448.0
    table = (w.rope_np * np.float32(1.37)).astype(np.float32)
    w.append([200], poke=poke)
    d = Stream(torch, KV, 2, 128, 64, [200], 32)
    moves = KV.KVMoves(i32(torch, [0, 200]), i32(torch, range(200)), i32(torch, [0]), i32(torch, w.table), i32(torch, d.table), 200)
    d.cache.compact(moves, rope=KV.Rope(torch.from_numpy(table).to(DEV)), source=w.cache)
    d.held = np.array([200])
    old, new = w.rows(0), d.rows(0)
    assert np.array_equal(old[0], new[0]) and np.array_equal(old[1], new[1])
    for x, byte in ((old[0], new[2]), (old[1], new[3])):
        assert all(byte[i, h] == K.scale_byte(np.abs(x[i // 32 * 32:i // 32 * 32 + 32, h]).max()) for i in range(200) for h in range(2))


def test_turning_there_and_back_with_scaled_tables(torch, KV):
    """A table whose rows have different sizes: keys are divided by the old one's and multiplied by the new one's."""
    w = Stream(torch, KV, 1, 64, 32, [300], 33, dims=64)
    w.append([300])
    size = (1.0 + np.arange(w.rope_np.shape[0]) % 5)[:, None].astype(np.float32)
    table = w.rope_np * size
    old = w.rows(0)
    tokens = np.arange(7, 300, 2)
    d = Stream(torch, KV, 1, 64, 32, [200], 34)
    moves = KV.KVMoves(i32(torch, [0, len(tokens)]), i32(torch, tokens), i32(torch, [0]), i32(torch, w.table), i32(torch, d.table), len(tokens))
    d.cache.compact(moves, rope=KV.Rope(torch.from_numpy(table).to(DEV)), source=w.cache)
    d.held = np.array([len(tokens)])
    none = (np.zeros((0, 1, 64)),) * 2 + (np.zeros((0, 1), int),) * 2
    check(old, d.rows(0), 0, tokens, table, False, 1, none)


@pytest.mark.parametrize("staged", [False, True])
def test_tokens_that_are_not_there_are_loud(torch, KV, staged):
    """Numbers outside the sequence, pages that the table does not name, NaN: NaN codes and zeros there, and nowhere else."""
    w = Stream(torch, KV, 2, 128, 32, [200], 35, dims=128)

    def poke(x):
        x[50, 2, 3] = float("nan")      # key of head 0
        x[60, 5, 9] = float("inf")      # value of head 1
    w.append([200], poke=poke)
    d = Stream(torch, KV, 2, 128, 64, [100], 36)
    tokens = np.concatenate([[-1, 2 ** 31 - 1, -2 ** 31, w.width * 32, 50, 60], np.arange(100, 120), [70], np.arange(120, 150)])
    table = w.table.copy()
    table[0, 70 // 32] = -1
    table[0, 50 // 32] = w.table[0, 50 // 32]
    moves = KV.KVMoves(i32(torch, [0, len(tokens)]), i32(torch, tokens), i32(torch, [3]), i32(torch, table), i32(torch, d.table), len(tokens))
    d.append([3])
    d.cache.compact(moves, rope=w.rope, source=w.cache, workspace=d.cache.compact_workspace(moves) if staged else None)
    torch.cuda.synchronize()
    d.held = np.array([3 + len(tokens)])
    k, v, _, _ = d.rows(0)
    gone = np.zeros((3 + len(tokens), 2), bool)
    gone[3:7] = gone[3 + 26] = True
    gone[7, 0] = gone[8, 1] = True
    assert np.array_equal(np.isnan(k).all(-1), gone) and np.array_equal(np.isnan(k).any(-1), gone) and (v[gone] == 0).all() and np.isfinite(v).all()
    good = np.flatnonzero(~gone.any(1))[3:]
    old_v = w.rows(0)[1]
    assert np.allclose(v[good], old_v[tokens[good - 3]], rtol=2.0 ** -4, atol=1e-2)


def test_tables_and_counts_out_of_range_touch_nothing(torch, KV):
    w = Stream(torch, KV, 2, 64, 32, [64, 64], 37)
    w.append([64, 64])
    d = Stream(torch, KV, 2, 64, 32, [64, 64], 38)
    keep = [t.clone() for t in d.buffers()]
    tokens = np.tile(np.arange(40), 2)
    for staged in (False, True):
        for table in (np.full((2, 2), -1), np.full((2, 2), d.pages), np.full((2, 2), 2 ** 31 - 1)):
            moves = KV.KVMoves(i32(torch, [0, 40, 80]), i32(torch, tokens), i32(torch, [0, 5]), i32(torch, w.table), i32(torch, table), 80)
            d.cache.compact(moves, source=w.cache, workspace=d.cache.compact_workspace(moves) if staged else None)
        moves = KV.KVMoves(i32(torch, [0, 40, 80]), i32(torch, tokens), i32(torch, [64, 2 ** 31 - 1]), i32(torch, w.table), i32(torch, d.table), 80)      # past the pages
        d.cache.compact(moves, source=w.cache, workspace=d.cache.compact_workspace(moves) if staged else None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(keep, d.buffers()))
        for cu in ([0, 60, 20], [5, 200, 90], [-9, -3, 400], [80, 80, 80]):      # clamped
            for first in ([0, 5], [-7, 60], [-2 ** 31, 2 ** 31 - 1]):
                moves = KV.KVMoves(i32(torch, cu), i32(torch, tokens), i32(torch, first), i32(torch, w.table), i32(torch, d.table), 80)
                d.cache.compact(moves, source=w.cache, workspace=d.cache.compact_workspace(moves) if staged else None)
        torch.cuda.synchronize()
        for t, s in zip(d.buffers(), keep):
            t.copy_(s)
