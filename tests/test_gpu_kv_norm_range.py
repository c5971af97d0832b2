"""Norms of keys and queries whose eps is not small beside squares that leave fp32: the factor is that of the definition in 64 bits, up to the largest eps that is taken."""
import numpy as np
import pytest

from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_streams import Stream, check_keys

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


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("eps,size", [(1e30, 2.0 ** 61), (1e36, 2.0 ** 60), (1e37, 2.0 ** 61), (1e38, 2.0 ** 64), (3.4e38, 2.0 ** 60), (3.4028234e38, 2.0 ** 20), (3.4e38, 2.0 ** 63)])
def test_squares_past_fp32_beside_a_large_eps(torch, KV, dim, eps, size):
    """Keys, queries of a few rows and of many; rows 1 and 40 are small ones among them."""
    w = Stream(torch, KV, 2, dim, 64, [200], 21, q_heads=4, dims=dim, norm=dict(first=5, eps=eps))

    def poke(x):
        x[:, :6] *= size                # queries and keys
        x[1::39, :6] *= 2.0 ** -50
    _, xn, _ = w.append([90], poke=poke)
    check_keys(w, [(xn[:, 4:6], xn[:, 6:], np.ones(90, bool))])
    for new in (3, 107):
        x, xn, _ = w.append([new], poke=poke)
        w.attend(x, xn, [new], scale=0.2)
