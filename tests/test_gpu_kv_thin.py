"""One branch of several is thinned out: its tokens go to pages that no other row names, so the others keep every byte.  The recipe of the interface's documentation, with a row that
begins anew and with one that goes on sharing the first tokens."""
import numpy as np
import pytest

from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_shortage import World, i32

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


@pytest.mark.parametrize("P,D,shared", [(64, 64, 0), (32, 128, 64), (64, 128, 75), (128, 64, 7)])
def test_a_branch_is_thinned_out_beside_others(torch, KV, P, D, shared):
    w = World(torch, KV, 60, P, D=D, seed=P + shared)
    t, c, fresh = w.rows(1, 8), w.rows(3, 8), w.rows(1, 8)
    w.step(t, [170])
    w.fork(t, [0, 0, 0], c)
    for new in ([1, 2, 3], [40, 20, 1]):
        w.step(c, new)
    # the branch's first tokens stay where they are, in pages that its new row shares; `kept` of the others go behind them, in pages of the row's own
    kept = shared + np.sort(w.rng.permutation(c.lens[1] - shared)[:80])
    old = w.held(c.host[1], np.arange(c.lens[1]))
    t2 = w.rows(1, 8)
    t2.copy_(c[1:2])
    t2.host, t2.lens = [list(c.host[1])], [shared]
    w.fork(t2, [0], fresh)      # (up to `shared` tokens)
    fresh.lens = [shared + 80]
    w.pool.reserve(w.cache, w.batch(fresh, [80]), w.missing)
    copies, missing = w.model.reserve(fresh.host, [80], fresh.lens)
    assert w.missing.item() == missing == 0 and fresh.tolist() == fresh.host and w.pool.refs.tolist() == w.model.refs
    buffers = (w.cache.k_codes, w.cache.k_scales, w.cache.v_codes, w.cache.v_scales)
    before, mine = [b.clone() for b in buffers], sorted({g for g in fresh.host[0][shared // P:] if g >= 0})
    assert all(w.model.refs[g] == 1 for g in mine)
    w.cache.compact(KV.KVMoves(i32(torch, [0, 80]), i32(torch, kept), i32(torch, [shared]), c[1:2].contiguous(), fresh, 80))
    others = np.setdiff1d(np.arange(60), mine)
    for a, b in zip(before, buffers):
        assert torch.equal(a[others.tolist()], b[others.tolist()])      # whatever is not the row's own
    got = w.held(fresh.host[0], np.arange(shared + 80))
    for side in (0, 1):
        moved = old[side][np.concatenate([np.arange(shared), kept])]
        byte = got[2 + side]
        assert (np.abs(got[side] - moved) <= W.code_bounds(moved, 0.0, byte[..., None]) + 2.0 ** -10 * np.exp2(np.maximum(byte, 1) - 127.0)[..., None]).all()
    # the old row ends, the new one and the others go on, each beside its own tokens
    fresh.have = [set(range(shared + 80))]
    fresh.sent = [{i: np.concatenate([got[0][i], got[1][i]]) for i in range(shared + 80)}]
    w.end((c, 1))
    w.step(fresh, [7])
    w.step(c, [1, 0, 9])
    w.end((c, 0), (c, 2), (fresh, 0), (t, 0))
    assert not w.pool.refs.any()
