"""An attention block with its keys and values in the paged 8-bit cache: quantized QKV layer, append, attention, quantized output layer.

    python examples/attention_block.py [--tokens 40] [--format int4|fp4|w8a8]

Three sequences share a pool of pages.  Their prompts are taken in ragged chunks, then a captured graph takes one token of each per replay.  The end compares
the block's attention with a softmax in 64 bits, over the keys and values as the cache holds them (read back by gather) and over those that went in.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2411_05007_amd import kv as KV  # noqa: E402
from paper_2411_05007_amd import svdq as S  # noqa: E402

DEV = "cuda:0"
HIDDEN, Q_HEADS, KV_HEADS, DIM, PAGE = 512, 8, 2, 64, 64
PREPARE = {"int4": (S.svdq_prepare, 32), "fp4": (S.svdq_fp4_prepare, 32), "w8a8": (S.svdq_w8a8_prepare, 16)}


class AttentionBlock:
    """out(attention(rotate(q), append(rotate(k), v))) for [q, k, v] = qkv(x)."""

    def __init__(self, fmt: str, positions: int, seed: int = 0):
        rng = np.random.default_rng(seed)
        prepare, rank = PREPARE[fmt]

        def layer(k, n):
            w = (rng.standard_normal((k, n)) * k ** -0.5 * 1.5).astype(np.float32)
            return S.DeviceLayer(prepare(w, np.full(k, 4.0, np.float32), rank), DEV)
        self.qkv, self.out = layer(HIDDEN, (Q_HEADS + 2 * KV_HEADS) * DIM), layer(Q_HEADS * DIM, HIDDEN)
        self.rope = KV.Rope(KV.rope_table(positions, DIM, device=DEV))

    def buffers(self, batch, cache):
        """What a call of a batch of this size writes to: kept by the caller from step to step."""
        T = batch.new_tokens
        new = lambda n: torch.empty(T, n, dtype=torch.bfloat16, device=DEV)
        return {"qkv": new(self.qkv.N), "attention": new(Q_HEADS * DIM).view(T, Q_HEADS, DIM), "y": new(HIDDEN), "qkv_ws": self.qkv.workspace(T),
                "attention_ws": cache.attention_workspace(batch, Q_HEADS), "out_ws": self.out.workspace(T)}

    def __call__(self, x, cache, batch, buf):
        q, k, v = KV.split_heads(self.qkv.forward(x, buf["qkv"], buf["qkv_ws"]), Q_HEADS, KV_HEADS)
        cache.append(k, v, batch, self.rope)
        a = cache.attention(q, batch, self.rope, out=buf["attention"], workspace=buf["attention_ws"])
        return self.out.forward(a.view(x.shape[0], -1), buf["y"], buf["out_ws"])


def rotated(x, pos, table):
    """x fp64 [tokens, heads, DIM] at positions pos"""
    c, s = table[pos, :DIM // 2][:, None], table[pos, DIM // 2:][:, None]
    a, b = x[..., :DIM // 2], x[..., DIM // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def softmax_attention(q, k, v, pos):
    """fp64, q [n, Q_HEADS, DIM] at positions pos, k and v [tokens, KV_HEADS, DIM]"""
    k, v = k.repeat_interleave(Q_HEADS // KV_HEADS, 1), v.repeat_interleave(Q_HEADS // KV_HEADS, 1)
    s = (q[:, None] * k[None]).sum(-1) * DIM ** -0.5
    s = s.masked_fill((torch.arange(k.shape[0], device=DEV)[None] > pos[:, None])[..., None], float("-inf"))
    return (s.softmax(1)[..., None] * v[None]).sum(1)


def main(tokens: int = 40, fmt: str = "int4", verbose: bool = True):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    chunks = [[70, 33, 1], [129, 0, 64], [1, 90, 40]]      # new tokens of the three sequences, chunk by chunk
    B = 3
    most = max(sum(c[b] for c in chunks) for b in range(B)) + tokens
    width = (most + PAGE - 1) // PAGE
    block = AttentionBlock(fmt, most)
    cache = KV.KVCache(B * width, KV_HEADS, DIM, PAGE)
    table = torch.randperm(B * width, generator=gen, device=DEV).int().view(B, width)
    seen = [[] for _ in range(B)]      # qkv rows of each sequence, for the comparison
    last = [None] * B
    held = [0] * B

    def note(buf, counts):
        at = 0
        for b, n in enumerate(counts):
            if n:
                seen[b].append(buf["qkv"][at:at + n].clone())
                last[b] = buf["attention"][at:at + n].clone()
            at += n

    for new in chunks:
        held = [h + n for h, n in zip(held, new)]
        batch = KV.KVBatch(i32([0, *np.cumsum(new)]), i32(held), table, sum(new), max(new), max(held))
        buf = block.buffers(batch, cache)
        block(torch.randn(sum(new), HIDDEN, generator=gen, device=DEV).to(torch.bfloat16), cache, batch, buf)
        note(buf, new)

    # one token of each sequence per replay; the lengths are device memory that the graph counts up itself
    length = i32(held)
    batch = KV.KVBatch(i32(list(range(B + 1))), length, table, B, 1, most)
    buf, x = block.buffers(batch, cache), torch.zeros(B, HIDDEN, dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):      # (the first call of a kernel loads it; lengths of zero touch no page)
        block(x, cache, KV.KVBatch(batch.cu_new, i32([0] * B), table, B, 1, most), buf)
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
        note(buf, [1] * B)
    end.record()
    torch.cuda.synchronize()
    assert length.tolist() == [h + tokens for h in held]

    stored = [0.0, 0.0]      # largest relative errors, against the cache's own numbers and against the 16-bit ones
    rope = block.rope.table.double()
    for b in range(B):
        n = int(length[b])
        k8, v8 = (t.double() for t in cache.gather(KV.KVRows(i32([0]), i32([0, n]), table[b:b + 1].contiguous(), n)))
        q, k, v = (t.double() for t in KV.split_heads(torch.cat(seen[b]), Q_HEADS, KV_HEADS))
        pos = torch.arange(n, device=DEV)
        got = last[b].double()
        where = pos[n - got.shape[0]:]
        q, k = rotated(q[where], where, rope), rotated(k, pos, rope)
        for i, (kk, vv) in enumerate(((k8, v8), (k, v))):
            want = softmax_attention(q, kk, vv, where)
            stored[i] = max(stored[i], float((got - want).norm() / want.norm()))
    if verbose:
        us = start.elapsed_time(end) * 1e3 / max(tokens, 1)
        print(f"{fmt}: {B} sequences of {[int(n) for n in length]} tokens, {us:.1f} us a step (with the copies for the comparison); attention's relative error "
              f"{stored[0]:.4f} over the cache's numbers, {stored[1]:.4f} over the 16-bit ones")
    return stored


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, default=40)
    a.add_argument("--format", choices=sorted(PREPARE), default="int4")
    args = a.parse_args()
    main(args.tokens, args.format)
