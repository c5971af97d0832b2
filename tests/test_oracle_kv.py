"""The oracle of the 8-bit cache against closed forms, and the entry points' refusals (no GPU takes part: every call returns before a launch)."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import kv_oracle as K
from paper_2411_05007_amd import svdq as S


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(S.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return S.lib()


def test_codes_stand_for_the_format_s_numbers():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(K.VALUES, want, equal_nan=True)


def test_rounding_takes_the_nearest_number_and_ties_go_to_the_even_code():
    grid = np.sort(K.VALUES[np.isfinite(K.VALUES) & ~np.signbit(K.VALUES)])
    codes = {float(K.VALUES[c]): c for c in range(127)}
    for a, b in zip(grid[:-1], grid[1:]):
        mid = (a + b) / 2
        assert K.e4m3_round(mid) == (a if codes[float(a)] % 2 == 0 else b)
        assert K.e4m3_round(mid * (1 - 1e-12)) == a and K.e4m3_round(mid * (1 + 1e-12)) == b
    assert np.array_equal(K.e4m3_round(grid), grid) and np.array_equal(K.e4m3_round(-grid), -grid)


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0 * (1 + 2.0 ** -23), 1), (1.75, -8), (1.7500002, -7), (2.0 ** -130, -126), (3.0e38, 120)])
def test_scale_byte_is_the_smallest_that_holds_the_block(amax, e):
    assert K.scale_byte(np.float32(amax)) == e + 127
    assert K.scale_byte(0.0) == 0


def test_rotation_keeps_lengths_and_differences_of_positions():
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 1, 64)).astype(np.float32)
    a = np.arange(40)[:, None] * 10000.0 ** (-np.arange(32) / 32.0)
    table = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)
    for inter in (False, True):
        assert np.isclose((K.rotate(x, 7, table, inter) ** 2).sum(), (x ** 2).sum(), rtol=1e-5)
        near = (K.rotate(x, 30, table, inter) * K.rotate(y, 28, table, inter)).sum()
        far = (K.rotate(x, 9, table, inter) * K.rotate(y, 7, table, inter)).sum()
        assert np.isclose(near, far, atol=1e-4)


def test_a_block_filled_in_pieces_ends_with_the_scale_of_the_whole():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal((40, 2, 64)) * np.exp2(np.arange(40) / 8.0)[:, None, None]).astype(np.float32)
    whole, pieces = K.Cache(2, 64), K.Cache(2, 64)
    whole.append(0, 0, x, x)
    for a, b in ((0, 1), (1, 13), (13, 40)):
        pieces.append(0, a, x[a:b], x[a:b])
    for blk in (0, 1):
        assert np.array_equal(whole.k[0, blk][0], pieces.k[0, blk][0])
    # rounding twice differs from rounding once by a step of the format's subnormal numbers at most
    w, p = whole.rows(0, 0, 40)[0], pieces.rows(0, 0, 40)[0]
    top = np.exp2(whole.k[0, 0][0].astype(float) - 127)[None, :, None] * 2.0 ** -9
    assert np.all(np.abs(w - p)[:32] <= top) and np.array_equal(w[32:], p[32:])


def test_attention_is_the_softmax_of_the_scores():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 4, 16)), rng.standard_normal((9, 2, 16)), rng.standard_normal((9, 2, 16))
    out, _ = K.attention(q, k, v, np.arange(4, 9), 0.25, True, 3)
    t = lambda x: torch.from_numpy(x).permute(1, 0, 2)
    j, i = torch.arange(9), torch.arange(4, 9)[:, None]
    mask = (j <= i) & (j > i - 3)
    want = torch.nn.functional.scaled_dot_product_attention(t(q), t(k).repeat_interleave(2, 0), t(v).repeat_interleave(2, 0), attn_mask=mask, scale=0.25)
    assert np.allclose(out, want.permute(1, 0, 2).numpy(), atol=1e-12)
    assert np.array_equal(K.attention(q, k, v, np.arange(-9, -4), 0.25, True, 0)[0], np.zeros((5, 4, 16)))


# ---- refusals: pointers are never followed, the checks come first --------------------------------------------------------------------------

AT = 0x10000000


def _good():
    cache = S.KVCacheDev(AT, AT, AT, AT, 4, S.KVShape(2, 128, 64))
    batch = S.KVBatchDev(AT, AT, AT, 3, 2, 5, 4, 100)
    rope = S.KVRopeDev(AT, 100, 128, 0)
    rows = S.KVRowsDev(AT, 6 * 128, 128)
    return cache, batch, rope, rows


def _set(path, value):
    def change(a):
        o = a[path[0]]
        for n in path[1:-1]:
            o = getattr(o, n)
        setattr(o, path[-1], value)
    return change


CACHE, BATCH, ROPE, ROWS = range(4)
COMMON = [(_set((CACHE, "k_codes"), None), -1), (_set((CACHE, "v_scales"), None), -1), (_set((CACHE, "v_codes"), AT + 8), -1), (_set((CACHE, "pages"), 0), -1),
          (_set((CACHE, "shape", "kv_heads"), 0), -1), (_set((CACHE, "shape", "head_dim"), 96), -2), (_set((CACHE, "shape", "page_tokens"), 48), -2),
          (_set((CACHE, "shape", "page_tokens"), 16), -2), (_set((CACHE, "shape", "page_tokens"), 2048), -2), (_set((CACHE, "shape", "kv_heads"), 70000), -2)]
BATCHED = [(_set((BATCH, "cu_new"), None), -1), (_set((BATCH, "kv_len"), AT + 2), -1), (_set((BATCH, "block_table"), None), -1), (_set((BATCH, "sequences"), -1), -1),
           (_set((BATCH, "new_tokens"), -1), -1), (_set((BATCH, "table_width"), 0), -1), (_set((BATCH, "sequences"), 70000), -2), (_set((BATCH, "table_width"), 1 << 25), -2),
           (_set((ROPE, "table"), None), -1), (_set((ROPE, "table"), AT + 4), -1), (_set((ROPE, "dims"), 24), -1), (_set((ROPE, "dims"), 256), -1), (_set((ROPE, "positions"), 0), -1),
           (_set((ROWS, "data"), None), -1), (_set((ROWS, "data"), AT + 2), -1), (_set((ROWS, "token_stride"), 129), -1), (_set((ROWS, "head_stride"), 4), -1)]


@pytest.mark.parametrize("i", range(len(COMMON + BATCHED)))
def test_append_refuses(lib, i):
    change, want = (COMMON + BATCHED)[i]
    a = _good()
    change(a)
    assert lib.svdq_kv_append(a[0], a[1], a[2], a[3], a[3], None) == want


def _attend(lib, a, q_heads=4, window=0, out=AT, ws=AT, n=1 << 40):
    return lib.svdq_kv_attention(a[0], a[1], a[2], a[3], q_heads, 0.1, 1, window, out, ws, n, None)


@pytest.mark.parametrize("i", range(len(COMMON + BATCHED)))
def test_attention_refuses(lib, i):
    change, want = (COMMON + BATCHED)[i]
    a = _good()
    change(a)
    assert _attend(lib, a) == want


@pytest.mark.parametrize("kw,want", [({"q_heads": 3}, -1), ({"q_heads": 0}, -1), ({"window": -1}, -1), ({"out": None}, -1), ({"out": AT + 8}, -1), ({"ws": None}, -1),
                                     ({"ws": AT + 16}, -1)])
def test_attention_refuses_its_own_arguments(lib, kw, want):
    assert _attend(lib, _good(), **kw) == want


def test_attention_refuses_a_small_workspace_and_sizes_past_its_grid(lib):
    a = _good()
    a[1].max_len, a[1].max_new, a[1].table_width = 60000, 1, 1000
    n = lib.svdq_kv_attention_workspace_bytes(C.byref(a[0].shape), 4, 3, 1, 60000)
    assert n > 256
    assert _attend(lib, a, n=n - 1) == -4
    a[1].max_len = 1 << 30 | 1
    assert _attend(lib, a) == -2
    for bad in ((S.KVShape(2, 96, 64), 4, 3, 1, 10), (S.KVShape(2, 128, 64), 3, 3, 1, 10), (S.KVShape(2, 128, 64), 4, -1, 1, 10), (S.KVShape(2, 128, 64), 4, 3, -1, 10),
                (S.KVShape(2, 128, 64), 4, 3, 1, -1)):
        assert lib.svdq_kv_attention_workspace_bytes(C.byref(bad[0]), *bad[1:]) == 0


@pytest.mark.parametrize("i", range(len(COMMON)))
def test_gather_and_sizes_refuse(lib, i):
    change, want = COMMON[i]
    a = _good()
    change(a)
    assert lib.svdq_kv_gather(a[0], AT, AT, AT, 3, 2, 5, AT, AT, None) == want
    good = _good()[0]
    for args in ((None, AT, AT, 3, 2, 5, AT, AT), (AT, AT, AT, -3, 2, 5, AT, AT), (AT, AT, AT, 3, 2, -5, AT, AT), (AT, AT, AT, 3, 2, 5, AT + 2, AT)):
        assert lib.svdq_kv_gather(good, *args, None) == -1
    sizes = S.KVSizes()
    assert lib.svdq_kv_cache_sizes(C.byref(S.KVShape(2, 128, 64)), 0, C.byref(sizes)) == -1
    assert lib.svdq_kv_cache_sizes(C.byref(S.KVShape(2, 72, 64)), 1, C.byref(sizes)) == -2
    assert lib.svdq_kv_cache_sizes(C.byref(S.KVShape(2, 128, 64)), 3, C.byref(sizes)) == 0 and (sizes.codes, sizes.scales) == (3 * 2 * 64 * 128, 3 * 2 * 2)


def test_empty_calls_do_nothing(lib):
    a = _good()
    a[1].new_tokens = 0
    assert lib.svdq_kv_append(a[0], a[1], a[2], None, None, None) == 0 and _attend(lib, a) == 0
    a[1].new_tokens, a[1].sequences = 5, 0
    assert lib.svdq_kv_append(a[0], a[1], a[2], None, None, None) == 0 and _attend(lib, a) == 0
    assert lib.svdq_kv_gather(a[0], None, None, None, 0, 0, 0, AT, AT, None) == 0
