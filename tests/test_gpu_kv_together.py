"""Streams, branches and compaction as a program uses them together: prompts, steps in a captured graph that keeps within a few pages, branches that go their own way, one that is thinned
out and goes on.  Attention is held to the definition in 64 bits over what the cache holds, step by step."""
import numpy as np
import pytest

from oracle import kv_stream_oracle as W
from paper_2411_05007_amd import svdq as S
from tests.test_gpu_kv_compact import check
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


class Program:
    """Sequences in rows of a table whose pages a pool hands out."""

    def __init__(self, torch, KV, pages, rows, width, H=2, G=2, D=128, P=64, window=100, sinks=5, seed=1):
        self.torch, self.KV, self.H, self.G, self.D, self.P, self.window, self.sinks = torch, KV, H, G, D, P, window, sinks
        self.w = Stream(torch, KV, H, D, P, [width * P] * rows, seed, q_heads=H * G, dims=D, interleaved=True, norm=dict(first=7), positions=width * P + 1)
        self.w.cache = KV.KVCache(pages, H, D, P)
        for t in self.w.buffers():
            t.fill_(0xFF)
        self.pool = KV.KVPages(pages, P)
        self.table = torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
        self.length, self.end = i32(torch, [0] * rows), i32(torch, [0] * rows)
        self.first = i32(torch, [(sinks + P - 1) // P * P] * rows)
        self.missing = i32(torch, [0])
        self.gen = torch.Generator(device=DEV).manual_seed(seed)

    def rows(self, n):
        return self.torch.randn(n, (self.G + 2) * self.H, self.D, generator=self.gen, device=DEV).to(self.torch.bfloat16)

    def step(self, x, batch, out=None, workspace=None, pages=None):
        """What a step is: pages, keys and values, attention, and the pages that the window has left."""
        q, k, v = x[:, :self.G * self.H], x[:, self.G * self.H:self.G * self.H + self.H], x[:, self.G * self.H + self.H:]
        self.pool.reserve(self.w.cache, batch, self.missing, workspace=pages)
        self.w.cache.append(k, v, batch, self.w.rope, norm=self.w.norm.dev)
        out = self.w.cache.attention(q, batch, self.w.rope, window=self.window, sinks=self.sinks, norm=self.w.norm.dev, out=out, workspace=workspace)
        self.torch.sub(batch.kv_len, self.window - 1, out=self.end[:batch.sequences])      # the next token sees what lies behind it
        self.pool.release(batch.block_table, self.first[:batch.sequences], self.end[:batch.sequences])
        return out

    def batch(self, new, lens, table=None, most=None):
        cu = np.concatenate([[0], np.cumsum(new)])
        return self.KV.KVBatch(i32(self.torch, cu), i32(self.torch, lens), self.table if table is None else table, int(cu[-1]), int(max(new)), int(most or max(lens)))

    def held(self, row, n):
        """keys and values of a row's tokens as its pages hold them, and which tokens those are"""
        self.w.table, self.w.held = np.where(row >= 0, row, 0)[None], np.array([n])
        k, v, _, _ = self.w.rows(0)
        there = np.repeat(row >= 0, self.P)[:n]
        return k[there], v[there], np.flatnonzero(there)

    def check(self, x, out, row, n, new):
        """out of a sequence's `new` last tokens; the window and the first tokens are held, whatever was given back"""
        k, v, keys = self.held(row, n)
        at = n - new + np.arange(new)
        assert all(W.seen(at, np.arange(n), True, self.window, self.sinks).any(0)[np.setdiff1d(np.arange(n), keys)] == False)  # noqa: E712
        q, size = self.w.norm.ready(x[:, :self.G * self.H].float().cpu().numpy(), at, "q", self.w.rope_np, True)
        want, tol = W.attention(q, size, k, v, at, keys, self.D ** -0.5, True, self.window, self.sinks)
        assert (np.abs(out.float().cpu().numpy() - want) <= tol).all()


def test_a_stream_in_a_few_pages(torch, KV):
    """Three sequences of up to 500 tokens in 13 pages of 64: a window of 100 and five first tokens need four pages each, a step one more."""
    p = Program(torch, KV, 13, 3, 9)
    lens = np.array([150, 20, 90])
    # prompts by chunks, pages given back between them
    done = np.zeros(3, int)
    for new in ([60, 20, 40], [60, 0, 50], [30, 0, 0]):
        done += new
        x, batch = p.rows(sum(new)), p.batch(new, done)
        before = p.table.clone()
        out = p.step(x, batch)
        assert p.missing.item() == 0
        at = 0
        for b, n in enumerate(new):
            if n:      # (the pages of the step were there during it)
                p.check(x[at:at + n], out[at:at + n], np.maximum(p.table[b].cpu().numpy(), before[b].cpu().numpy()), int(done[b]), n)
            at += n
    assert (done == lens).all()
    # one token of each a replay
    p.length.copy_(i32(torch, lens))
    batch = KV.KVBatch(i32(torch, range(4)), p.length, p.table, 3, 1, 9 * 64)
    x, out = p.rows(3), torch.empty(3, p.G * p.H, p.D, dtype=torch.bfloat16, device=DEV)
    ws, pages = p.w.cache.attention_workspace(batch, p.G * p.H), p.pool.reserve_workspace(batch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    idle = KV.KVBatch(i32(torch, [0] * 4), i32(torch, [0] * 3), torch.full_like(p.table, -1), 3, 1, 9 * 64)      # (the first call of a kernel loads it; no tokens)
    with torch.cuda.stream(side):
        p.step(x, idle, out, ws, pages)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.length.add_(1)
        p.step(x, batch, out, ws, pages)
    most = 0
    for i in range(350):
        x.copy_(p.rows(3))
        before = p.table.cpu().numpy()
        graph.replay()
        if i % 29 == 0 or i > 345:
            torch.cuda.synchronize()
            lens = p.length.tolist()
            assert p.missing.item() == 0 and lens == [150 + i + 1, 20 + i + 1, 90 + i + 1]
            most = max(most, int((p.pool.refs > 0).sum()))
            for b in range(3):
                p.check(x[b:b + 1], out[b:b + 1], np.maximum(p.table[b].cpu().numpy(), before[b]), lens[b], 1)
    assert most <= 12 and int(p.pool.refs.sum()) == int((p.table >= 0).sum())
    p.pool.release(p.table)
    assert not p.pool.refs.any()


def test_branches_and_a_sequence_that_is_thinned_out(torch, KV):
    """Two prompts, three branches of each (one of which the prompt's own row becomes), tokens of their own; one is thinned out to pages of its own and goes on, the others end."""
    p = Program(torch, KV, 60, 2, 8, window=10 ** 6, sinks=0)
    x = p.rows(290)
    p.step(x, p.batch([170, 120], [170, 120]))
    table, lens = torch.full((6, 8), -1, dtype=torch.int32, device=DEV), i32(torch, [0] * 6)
    p.pool.fork(p.table, i32(torch, [170, 120]), i32(torch, [0, 0, 0, 1, 1, 1]), table, lens)
    p.pool.release(p.table)
    n = [170] * 3 + [120] * 3
    p.first, p.end = i32(torch, [0] * 6), i32(torch, [0] * 6)
    for new in ([1, 2, 3, 1, 1, 1], [40, 1, 1, 1, 70, 1], [1] * 6):
        n = [a + b for a, b in zip(n, new)]
        x = p.rows(sum(new))
        out = p.step(x, p.batch(new, n, table))
        rows, at = table.cpu().numpy(), 0
        assert p.missing.item() == 0
        for b in range(6):
            p.check(x[at:at + new[b]], out[at:at + new[b]], rows[b], n[b], new[b])
            at += new[b]
    assert (p.pool.refs[table[:3, 0].long()] == 3).all() and (table[0, 0] == table[2, 0]).item()
    # branch 4 keeps its first 30 tokens and half of the others, in pages of its own
    rng = np.random.default_rng(3)
    keep = np.concatenate([np.arange(30), 30 + np.sort(rng.permutation(n[4] - 30)[:80])])
    thin = torch.full((1, 8), -1, dtype=torch.int32, device=DEV)
    p.pool.reserve(p.w.cache, p.batch([110], [110], thin), p.missing)
    row = table[4].cpu().numpy()
    p.w.table, p.w.held = np.where(row >= 0, row, 0)[None], np.array([n[4]])
    old = p.w.rows(0)
    source = table[4:5].contiguous()
    p.w.cache.compact(KV.KVMoves(i32(torch, [0, 110]), i32(torch, keep), i32(torch, [0]), source, thin, 110), rope=p.w.rope)
    p.w.table, p.w.held = np.maximum(thin.cpu().numpy(), 0), np.array([110])
    none = (np.zeros((0, 2, 128)),) * 2 + (np.zeros((0, 2), int),) * 2
    check(old, p.w.rows(0), 0, keep, p.w.rope_np, True, 2, none)
    p.pool.release(table)
    assert int(p.pool.refs.sum()) == 2
    # and goes on: a window now, pages given back
    p.window, p.sinks, p.first = 40, 3, i32(torch, [64])
    length = 110
    for new in (1, 17, 1, 90, 1):
        length += new
        x, before = p.rows(new), thin.cpu().numpy()
        out = p.step(x, p.batch([new], [length], thin))
        assert p.missing.item() == 0
        p.check(x, out, np.maximum(thin[0].cpu().numpy(), before[0]) if new == 1 else np.where(before[0] >= 0, before[0], thin[0].cpu().numpy()), length, new)
    p.pool.release(thin)
    assert not p.pool.refs.any()
