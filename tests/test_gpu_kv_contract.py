"""What include/svdq.h says of batches that do not fit their own description, of workspaces and of streams, in attention over the paged 8-bit cache."""
import numpy as np
import pytest

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


def filled(torch, KV, heads, dim, tokens, page=64, seed=1):
    """a cache that holds `tokens` random tokens in order, and its block table"""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    x = torch.randn(tokens, 2 * heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
    pages = (tokens + page - 1) // page
    cache, table = KV.KVCache(pages, heads, dim, page), torch.arange(pages, dtype=torch.int32, device=DEV)[None].contiguous()
    cache.append(x[:, :heads], x[:, heads:], KV.KVBatch(i32(torch, [0, tokens]), i32(torch, [tokens]), table, tokens, tokens, tokens))
    return cache, table


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,new,length,copies", [
    (64, 3, 1, 1), (128, 40, 33, 1), (256, 5, 0, 2),            # few rows
    (64, 200, 150, 512), (128, 200, 1, 512), (128, 200, 0, 300), (256, 140, 70, 512),      # many
    (128, 2000, 1500, 1),                                       # in parts
])
def test_tokens_without_a_position_see_no_key(torch, KV, dim, new, length, copies, causal):
    cache, table = filled(torch, KV, 1, dim, 2048)
    group = 8 if new == 2000 else 2
    q = torch.randn(new, group, dim, device=DEV).to(torch.bfloat16)
    batch = lambda n: KV.KVBatch(i32(torch, np.arange(copies + 1) * n), i32(torch, [length] * copies), table.expand(copies, -1).contiguous(), copies * n, n, length)
    out = cache.attention(q.repeat(copies, 1, 1), batch(new), causal=causal).view(copies, new, group, dim)
    without = new - length
    assert bool((out[:, :without] == 0).all())
    if length:      # the others are as they are alone (another cut of the rows: two roundings of an output at most)
        alone = cache.attention(q[without:].repeat(copies, 1, 1), batch(length), causal=causal).view(copies, length, group, dim)
        assert float((out[:, without:].float() - alone.float()).abs().max()) <= 2.0 ** -7 * float(alone.float().abs().max())
        assert bool((alone != 0).any(-1).all())
