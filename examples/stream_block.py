"""An attention block that streams: quantized QKV layer, norms of heads, a window with first tokens that stay visible, pages handed out and given back on the GPU.

    python examples/stream_block.py [--tokens 600] [--format int4|fp4|w8a8]

Two sequences take their prompts, each branches in two, and all four go on for as many tokens as asked, one of each per replay of a captured graph that counts lengths, reserves pages, appends,
attends and gives pages back by itself.  The pool holds a few pages for each sequence, however long they get.  The end compares the last step with a softmax in 64 bits over what the cache holds.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from examples.attention_block import DEV, DIM, HIDDEN, KV_HEADS, PAGE, PREPARE, Q_HEADS, AttentionBlock, rotated  # noqa: E402
from paper_2411_05007_amd import kv as KV  # noqa: E402

WINDOW, SINKS, EPS = 128, 4, 1e-6


class StreamBlock(AttentionBlock):
    """The block with normalised heads in a window, its pages kept by a pool."""

    def __init__(self, fmt: str, positions: int, pool: KV.KVPages, seed: int = 0):
        super().__init__(fmt, positions, seed)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.q_weight, self.k_weight = (0.5 + torch.rand(DIM, generator=gen, device=DEV) for _ in range(2))
        self.norm, self.pool = KV.KVNorm(self.q_weight, self.k_weight, EPS), pool

    def buffers(self, batch, cache):
        B, i32 = batch.sequences, dict(dtype=torch.int32, device=DEV)
        return {**super().buffers(batch, cache), "pages_ws": self.pool.reserve_workspace(batch), "missing": torch.zeros(1, **i32), "lost": torch.zeros(1, **i32),
                "first": torch.full((B,), (SINKS + PAGE - 1) // PAGE * PAGE, **i32), "end": torch.zeros(B, **i32)}

    def __call__(self, x, cache, batch, buf):
        q, k, v = KV.split_heads(self.qkv.forward(x, buf["qkv"], buf["qkv_ws"]), Q_HEADS, KV_HEADS)
        self.pool.reserve(cache, batch, buf["missing"], workspace=buf["pages_ws"])
        buf["lost"].add_(buf["missing"])      # of all steps: each writes `missing` anew
        cache.append(k, v, batch, self.rope, norm=self.norm)
        a = cache.attention(q, batch, self.rope, window=WINDOW, sinks=SINKS, norm=self.norm, out=buf["attention"], workspace=buf["attention_ws"])
        torch.sub(batch.kv_len, WINDOW - 1, out=buf["end"])      # the next token's window begins there
        self.pool.release(batch.block_table, buf["first"], buf["end"])
        return self.out.forward(a.view(x.shape[0], -1), buf["y"], buf["out_ws"])


def main(tokens: int = 600, fmt: str = "int4", verbose: bool = True):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    prompts, branches = [90, 200], 2
    B, most = len(prompts) * branches, max(prompts) + tokens
    width = (most + PAGE - 1) // PAGE
    # a sequence holds the pages of its first tokens and of its window, and one more during a step; a prompt is taken whole
    pages = max(B * (1 + (WINDOW + PAGE - 2) // PAGE + 2), sum((n + PAGE - 1) // PAGE for n in prompts) + B * 2)
    pool = KV.KVPages(pages, PAGE)
    cache, block = KV.KVCache(pages, KV_HEADS, DIM, PAGE), StreamBlock(fmt, most, pool)
    none = lambda rows: torch.full((rows, width), -1, dtype=torch.int32, device=DEV)
    parents = none(len(prompts))
    batch = KV.KVBatch(i32([0, prompts[0], sum(prompts)]), i32(prompts), parents, sum(prompts), max(prompts), max(prompts))
    buf = block.buffers(batch, cache)
    block(torch.randn(sum(prompts), HIDDEN, generator=gen, device=DEV).to(torch.bfloat16), cache, batch, buf)
    assert buf["lost"].item() == 0

    table, length = none(B), i32([0] * B)
    pool.fork(parents, i32(prompts), i32([b // branches for b in range(B)]), table, length)
    pool.release(parents)      # (the branches hold the pages now)
    batch = KV.KVBatch(i32(list(range(B + 1))), length, table, B, 1, most)
    buf, x = block.buffers(batch, cache), torch.zeros(B, HIDDEN, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):      # (the first call of a kernel loads it; sequences without tokens touch no page)
        block(x, cache, KV.KVBatch(i32([0] * (B + 1)), i32([0] * B), none(B), B, 1, most), buf)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        length.add_(1)
        block(x, cache, batch, buf)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    steps = torch.randn(tokens, B, HIDDEN, generator=gen, device=DEV).to(torch.bfloat16)
    start.record()
    for i in range(tokens):
        x.copy_(steps[i])
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    assert buf["lost"].item() == 0 and length.tolist() == [n + tokens for n in prompts for _ in range(branches)]

    error, rope = 0.0, block.rope.table.double()
    for b in range(B):
        n = int(length[b])
        seen = torch.cat([torch.arange(min(SINKS, n - WINDOW), device=DEV), torch.arange(n - WINDOW, n, device=DEV)]) if n > WINDOW else torch.arange(n, device=DEV)
        k, v = (t.double()[seen] for t in cache.gather(KV.KVRows(i32([0]), i32([0, n]), table[b:b + 1].contiguous(), n)))
        q = KV.split_heads(buf["qkv"][b:b + 1], Q_HEADS, KV_HEADS)[0].double()
        q = rotated(q / (q.square().mean(-1, keepdim=True) + EPS).sqrt() * block.q_weight.double(), torch.tensor([n - 1], device=DEV), rope)
        k, v = k.repeat_interleave(Q_HEADS // KV_HEADS, 1), v.repeat_interleave(Q_HEADS // KV_HEADS, 1)
        want = (((q * k).sum(-1) * DIM ** -0.5).softmax(0)[..., None] * v).sum(0)
        error = max(error, float((buf["attention"][b].double() - want).norm() / want.norm()))
    used = int((pool.refs > 0).sum())
    if verbose:
        print(f"{fmt}: {B} sequences of {length.tolist()} tokens in {used} of {pages} pages of {PAGE} ({sum(-(-n // PAGE) for n in length.tolist())} would hold all), "
              f"{start.elapsed_time(end) * 1e3 / max(tokens, 1):.1f} us a step; attention's relative error {error:.4f} over the cache's numbers")
    return error, used, pages


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, default=600)
    a.add_argument("--format", choices=sorted(PREPARE), default="int4")
    args = a.parse_args()
    main(args.tokens, args.format)
