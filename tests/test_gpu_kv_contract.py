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


@pytest.mark.parametrize("dim,group,max_new,new,length", [
    (128, 4, 1, 2, 500), (128, 4, 1, 2, 9000), (64, 1, 1, 3, 500), (64, 1, 1, 3, 9000), (256, 3, 2, 5, 5000), (128, 5, 3, 4, 9000), (64, 5, 4, 9, 700),
    (128, 4, 5, 300, 700),      # two tiles of rows
])
def test_tokens_past_the_most_leave_the_others_right(torch, KV, dim, group, max_new, new, length):
    """A sequence has more new tokens than the batch says that any has: the first ones are as they are in a batch that says it, the others like that or not written."""
    cache, table = filled(torch, KV, 2, dim, length, seed=3)
    q = torch.randn(new, 2 * group, dim, device=DEV).to(torch.bfloat16)
    batch = lambda most: KV.KVBatch(i32(torch, [0, new]), i32(torch, [length]), table, new, most, length)
    want = cache.attention(q, batch(new)).float()
    workspace = torch.full((cache.attention_workspace(batch(max_new), 2 * group).numel() + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
    for _ in range(3):
        guard = torch.full((new + 2, 2 * group, dim), 77.0, dtype=torch.bfloat16, device=DEV)
        cache.attention(q, batch(max_new), out=guard[1:-1], workspace=workspace[:-4096])
        torch.cuda.synchronize()
        assert bool((guard[[0, -1]] == 77).all()) and bool((workspace[-4096:] == 0x5A).all())
        got = guard[1:-1].float()
        right = (got - want).abs() <= 2.0 ** -7 * want.abs().max()      # (another cut: two roundings of an output at most)
        assert bool(right[:max_new].all())
        assert bool((right | (got == 77))[max_new:].all())


@pytest.mark.parametrize("dim,heads,sequences", [(64, 3, 5), (128, 2, 300), (256, 16, 40), (128, 8, 256)])
def test_both_halves_of_a_block_grow_with_its_scale(torch, KV, dim, heads, sequences):
    """17 to 31 tokens are in a block when a much louder one comes: the codes of all of them are rounded again to the new scale, whichever wavefront has them.  (One byte
    a block, read before it is written; checked through what gather reads, against the codes' own values.)"""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(dim + heads)
    cache, table = KV.KVCache(sequences, heads, dim, 32), torch.randperm(sequences, generator=gen, device=DEV).int()[:, None].contiguous()
    for held in (17, 24, 31):
        n = sequences * held
        x = torch.randn(n, 2 * heads, dim, generator=gen, device=DEV).to(torch.bfloat16)
        cu = np.arange(sequences + 1)
        cache.append(x[:, :heads], x[:, heads:], KV.KVBatch(i32(torch, cu * held), i32(torch, [held] * sequences), table, n, held, held))
        rows = KV.KVRows(i32(torch, [0] * sequences), i32(torch, cu * held), table, n)
        before = cache.gather(rows)
        loud = torch.full((sequences, 2 * heads, dim), 448.0 * 32, dtype=torch.bfloat16, device=DEV)      # (every block's byte becomes that of 2^5)
        cache.append(loud[:, :heads], loud[:, heads:], KV.KVBatch(i32(torch, cu), i32(torch, [held + 1] * sequences), table, sequences, 1, held + 1))
        for a, b, scales in zip(before, cache.gather(rows), (cache.k_scales, cache.v_scales)):
            assert bool((scales == 127 + 5).all())
            assert torch.equal(b.float(), (a.float() / 32).to(torch.float8_e4m3fn).float() * 32)


def test_memory_of_a_call_on_another_stream_is_not_what_this_one_still_writes(torch, KV):
    """The current stream has a temporary to write and has given it back; a call on an idle stream must not be handed that memory."""
    cache, table = filled(torch, KV, 2, 128, 9000, seed=5)
    q = torch.randn(1, 8, 128, device=DEV).to(torch.bfloat16)
    batch = KV.KVBatch(i32(torch, [0, 1]), i32(torch, [9000]), table, 1, 1, 9000)
    rows = KV.KVRows(i32(torch, [0]), i32(torch, [0, 9000]), table, 9000)
    want, held = cache.attention(q, batch), cache.gather(rows)
    n = cache.attention_workspace(batch, 8).numel()
    assert n > 4096      # (parts that meet)
    torch.cuda.synchronize()
    side, big = torch.cuda.Stream(), torch.randn(4096, 4096, device=DEV)
    for _ in range(3):
        for _ in range(8):
            big @ big      # (the current stream is busy for a while)
        for _ in range(2):
            for size in (n, want.numel() * 2, held[0].numel() * 2, held[0].numel() * 2):
                torch.full((size,), 0x41, dtype=torch.uint8, device=DEV)      # written behind that, and given back at once
        got, (k, v) = cache.attention(q, batch, stream=side), cache.gather(rows, stream=side)
        mine = cache.attention(q, batch, workspace=cache.attention_workspace(batch, 8, stream=side), stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(mine, want) and torch.equal(k, held[0]) and torch.equal(v, held[1])


def test_a_call_on_a_captured_stream_is_replayed(torch, KV):
    """Memory of a call inside a capture is the graph's, whether the stream is named or not."""
    cache, table = filled(torch, KV, 2, 64, 3000, seed=6)
    q = torch.randn(1, 4, 64, device=DEV).to(torch.bfloat16)
    batch = KV.KVBatch(i32(torch, [0, 1]), i32(torch, [3000]), table, 1, 1, 3000)
    cache.attention(q, batch)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = cache.attention(q, batch)
        named = cache.attention(q, batch, stream=torch.cuda.current_stream())
    for i in range(4):
        q.copy_(torch.randn(1, 4, 64, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        want = cache.attention(q, batch)
        torch.cuda.synchronize()
        assert torch.equal(here, want) and torch.equal(named, want)


@pytest.mark.parametrize("dim,heads,group", [(128, 8, 4), (64, 2, 8), (256, 1, 3)])
def test_one_workspace_serves_every_batch_within_its_own(torch, KV, dim, heads, group):
    cache, table = filled(torch, KV, heads, dim, 8300, seed=7)

    def batch(sequences, new, length):
        return KV.KVBatch(i32(torch, np.arange(sequences + 1) * new), i32(torch, [length] * sequences), table.expand(sequences, -1).contiguous(), sequences * new, new, length)
    workspace = cache.attention_workspace(batch(5, 120, 8277), heads * group)
    for sequences, new, length in ((1, 1, 8180), (5, 1, 8277), (2, 1, 4000), (3, 1, 4000), (1, 120, 8277), (5, 120, 8277), (4, 30, 8000), (1, 7, 5000), (2, 60, 1030), (3, 5, 2500)):
        q = torch.randn(sequences * new, heads * group, dim, device=DEV).to(torch.bfloat16)
        b = batch(sequences, new, length)
        assert torch.equal(cache.attention(q, b, workspace=workspace), cache.attention(q, b))


def test_gather_of_tokens_past_any_table_is_zeros(torch, KV):
    cache, table = filled(torch, KV, 2, 64, 200, seed=8)
    for first in (2 ** 31 - 1, 2 ** 31 - 40, 2 ** 30 + 5, 2 ** 30 - 7, 256):
        guard = [torch.full((104, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        cache.gather(KV.KVRows(i32(torch, [first, 0]), i32(torch, [0, 70, 100]), table.expand(2, -1).contiguous(), 100), out=[g[2:-2] for g in guard])
        held = cache.gather(KV.KVRows(i32(torch, [0]), i32(torch, [0, 30]), table, 30))
        for g, h in zip(guard, held):
            assert bool((g[:2] == 9).all()) and bool((g[-2:] == 9).all()) and bool((g[2:72] == 0).all()) and torch.equal(g[72:102], h)
