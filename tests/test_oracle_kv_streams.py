"""Pins of the oracle for streams and branches on the paged 8-bit cache (oracle/kv_stream_oracle.py), by hand or against kv_oracle."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import kv_stream_oracle as W


def test_a_norm_by_hand():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    assert np.allclose(W.normalise(x, None, 0.0), [[[1.2, 1.6, 0, 0]]], rtol=1e-15)
    assert np.allclose(W.normalise(x, [2.0, 0.5, 1, 1], 6.25 * 3), x * [2, 0.5, 1, 1] / 5, rtol=1e-15)
    assert np.allclose(W.normalise(np.array([[[1e30] * 4]]), None, 1e-6), 1.0) and (W.normalise(np.zeros((1, 1, 4)), None, 1e-6) == 0).all()


@pytest.mark.parametrize("inter", [False, True])
def test_turning_is_kv_oracles_and_goes_back(inter):
    rng = np.random.default_rng(1)
    a = np.arange(40)[:, None] * 10000.0 ** (-np.arange(8) * 2.0 / 16)
    table = np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32) * 1.5
    x = rng.standard_normal((6, 2, 24)).astype(np.float32)
    pos = np.array([0, 1, 5, 39, 40, 77])      # (past the table: its last row)
    y, size = W.turn(x.astype(np.float64), pos, table, inter)
    for i in range(6):
        assert np.abs(y[i] - K.rotate(x[i], pos[i], table, inter)).max() <= 2.0 ** -22 * size.max()
    assert np.allclose(W.turn(y, pos, table, inter, back=True)[0], x, rtol=1e-12)
    new = np.array([3, 1, 30, 0, 39, 2])
    k, slack = W.moved_key(y, pos, new, table, inter)
    assert np.allclose(k, W.turn(x.astype(np.float64), new, table, inter)[0], rtol=1e-12)
    assert (k[1] == y[1]).all() and (slack[1] == 0).all() and (slack[0, :, :16] > 0).all() and (slack[:, :, 16:] == 0).all()


def test_what_is_seen():
    got = W.seen([-1, 0, 3, 6], range(7), True, 2, 1).astype(int)
    assert got.tolist() == [[0] * 7, [1, 0, 0, 0, 0, 0, 0], [1, 0, 1, 1, 0, 0, 0], [1, 0, 0, 0, 0, 1, 1]]
    assert W.seen([2], range(4), True, 0, 3).tolist() == [[True, True, True, False]]
    assert W.seen([2], range(4), False, 1, 0).all() and not W.seen([-1], range(4), False, 1, 0).any()


def test_attention_is_kv_oracles():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    pos = np.array([6, 7, 8])
    for causal, window in ((True, 0), (True, 4), (False, 0)):
        want, tol = K.attention(q, k, v, pos, 0.3, causal, window)
        got, wide = W.attention(q, np.abs(q), k, v, pos, np.arange(9), 0.3, causal, window, 0)
        assert np.allclose(got, want, rtol=1e-12) and (wide >= 0.99 * tol).all()
    # with first tokens: as if the keys between were not there
    keep = [0, 1, 5, 6, 7, 8]
    got, _ = W.attention(q, np.abs(q), k, v, pos, np.arange(9), 0.3, True, 2, 2)
    want, _ = W.attention(q, np.abs(q), k[keep], v[keep], pos, np.array(keep), 0.3, True, 2, 2)
    assert np.allclose(got, want, rtol=1e-12)
    k[3], v[4] = np.nan, np.inf      # hidden
    assert np.allclose(W.attention(q, np.abs(q), k, v, pos, np.arange(9), 0.3, True, 2, 2)[0], want, rtol=1e-12)


def test_bounds_of_codes():
    assert W.code_bounds(np.array([3.0, 1e-9]), 0.0, 120).tolist() == [3.0 / 16, 2.0 ** -17]
    assert W.scale_bytes(448.0, 0.0) == {127} and W.scale_bytes(448.0, 1e-3) == {127, 128} and W.scale_bytes(0.0, 0.0) == {0}
    # a slack as large as the distance to the next code moves it by a step at most
    for x in np.linspace(16.0, 30.0, 300):
        assert abs(K.e4m3_round(x + 0.3) - x) <= W.code_bounds(np.array(x), 0.3, 127)


def test_pages_by_hand():
    p = W.Pages(6, 32)
    t = [[-1] * 3, [-1] * 3]
    assert p.reserve(t, [40, 0], [40, 0]) == ([(-1, -1, 0)] * 2, 0) and t == [[0, 1, -1], [-1] * 3] and p.refs == [1, 1, 0, 0, 0, 0]
    c, lens = [[9] * 2, [9] * 2, [9] * 2], [0] * 3
    p.fork(t, [40, 0], [0, 0, 5], c, lens)
    assert c == [[0, 1], [0, 1], [-1, -1]] and lens == [40, 40, 0] and p.refs == [3, 3, 0, 0, 0, 0]
    assert p.reserve(c, [1, 24, 1], [41, 64, 1]) == ([(1, 2, 8), (1, 3, 8), (-1, -1, 0)], 0)
    assert c == [[0, 2], [0, 3], [4, -1]] and p.refs == [3, 1, 1, 1, 1, 0]
    assert p.reserve(t, [57, 1], [97, 1]) == ([(-1, -1, 0)] * 2, 1) and t == [[0, 1, 5], [-1, -1, -1]]      # (97 tokens: the table holds 96; one page was left)
    p.release(c, [32, 0, 0], [64, 63, 32])
    assert c == [[0, -1], [-1, 3], [-1, -1]] and p.refs == [2, 1, 0, 1, 0, 1]
