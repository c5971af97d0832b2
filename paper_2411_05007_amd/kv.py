"""Binding of the paged 8-bit cache of keys and values and of the attention over it (``svdq_kv_*`` in ``include/svdq.h``).

    cache = KVCache(pages, kv_heads, head_dim, page_tokens)
    batch = KVBatch(cu_new, kv_len, block_table, new_tokens, max_new, max_len)
    q, k, v = split_heads(qkv, q_heads, kv_heads)                     # views of a QKV layer's output
    cache.append(k, v, batch, rope)                                   # keys rotated, both quantized
    out = cache.attention(q, batch, rope)                             # bf16 [tokens, q_heads, head_dim]

Argument marshalling only; every call enqueues on the current stream (or the one that is given) and does not synchronise.  A stream that is given is the caller's to order
behind what makes the inputs, and before what reads the results.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import svdq as S


_current_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else lambda i: torch.cuda.current_stream(i).cuda_stream


def _device_int32(t, name: str) -> None:
    assert t.dtype == torch.int32 and t.is_cuda and t.is_contiguous(), f"{name}: contiguous int32 on the GPU"


def split_heads(qkv, q_heads: int, kv_heads: int):
    """Queries, keys and values [tokens, heads, head_dim] of a fused QKV output [tokens, (q_heads + 2 kv_heads) * head_dim], as views."""
    x = qkv.view(qkv.shape[0], q_heads + 2 * kv_heads, -1)
    return x[:, :q_heads], x[:, q_heads:q_heads + kv_heads], x[:, q_heads + kv_heads:]


def rope_table(positions: int, dims: int, theta: float = 10000.0, device: str = "cuda:0"):
    """fp32 [positions, dims]: cosines and sines of p * theta^(-2 i / dims)."""
    i = torch.arange(dims // 2, dtype=torch.float64, device=device)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * torch.exp2(-math.log2(theta) * 2.0 / dims * i)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().contiguous()


class Rope:
    """A table of cosines and sines fp32 [positions, dims] and which channels it pairs: (i, i + dims / 2), or (2 i, 2 i + 1)."""

    def __init__(self, table, interleaved: bool = False):
        assert table.dtype == torch.float32 and table.is_cuda and table.is_contiguous() and table.dim() == 2
        self.table, self.interleaved = table, bool(interleaved)
        self.cdesc = S.KVRopeDev(table.data_ptr(), table.shape[0], table.shape[1], int(self.interleaved))


class KVBatch:
    """New tokens of some sequences.  cu_new int32 [B + 1], kv_len int32 [B] (tokens with the new ones), block_table int32 [B, width], all on the GPU;
    new_tokens = cu_new[B]; no sequence has more than max_new new tokens or more than max_len tokens."""

    def __init__(self, cu_new, kv_len, block_table, new_tokens: int, max_new: int, max_len: int):
        for t, n in ((cu_new, "cu_new"), (kv_len, "kv_len"), (block_table, "block_table")):
            _device_int32(t, n)
        B = kv_len.shape[0]
        assert cu_new.shape == (B + 1,) and block_table.dim() == 2 and block_table.shape[0] == B
        self.cu_new, self.kv_len, self.block_table = cu_new, kv_len, block_table
        self.sequences, self.new_tokens, self.max_new, self.max_len = B, int(new_tokens), int(max_new), int(max_len)
        self.cdesc = S.KVBatchDev(cu_new.data_ptr(), kv_len.data_ptr(), block_table.data_ptr(), B, block_table.shape[1], self.new_tokens, self.max_new, self.max_len)


class KVRows:
    """Rows to read back: of sequence b the tokens from first_token[b] on, cu_rows[b + 1] - cu_rows[b] of them."""

    def __init__(self, first_token, cu_rows, block_table, rows: int):
        for t, n in ((first_token, "first_token"), (cu_rows, "cu_rows"), (block_table, "block_table")):
            _device_int32(t, n)
        B = first_token.shape[0]
        assert cu_rows.shape == (B + 1,) and block_table.dim() == 2 and block_table.shape[0] == B
        self.first_token, self.cu_rows, self.block_table, self.sequences, self.rows = first_token, cu_rows, block_table, B, int(rows)
        self.pointers, self.width = (first_token.data_ptr(), cu_rows.data_ptr(), block_table.data_ptr()), block_table.shape[1]


class KVCache:
    """Pages of E4M3 codes with a scale byte for each 32 tokens and head, resident in HBM."""

    def __init__(self, pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise S.SvdqError("no GPU visible: the cache has no CPU path")
        sizes = S.KVSizes()
        shape = S.KVShape(kv_heads, head_dim, page_tokens)
        S._check(S.lib().svdq_kv_cache_sizes(C.byref(shape), int(pages), C.byref(sizes)), "svdq_kv_cache_sizes")
        zeros = lambda n: torch.zeros(n, dtype=torch.uint8, device=device)
        self._own(zeros(sizes.codes).view(pages, kv_heads, page_tokens // 32, 32, head_dim), zeros(sizes.scales).view(pages, kv_heads, page_tokens // 32),
                  zeros(sizes.codes).view(pages, kv_heads, page_tokens // 32, head_dim // 32, 16, 4, 2, 8), zeros(sizes.scales).view(pages, kv_heads, page_tokens // 32))

    @classmethod
    def from_buffers(cls, k_codes, k_scales, v_codes, v_scales) -> "KVCache":
        """A cache over buffers in the layout of ``include/svdq.h`` (uint8, e.g. of a saved cache); they are kept, not copied."""
        self = cls.__new__(cls)
        self._own(k_codes, k_scales, v_codes, v_scales)
        return self

    def _own(self, k_codes, k_scales, v_codes, v_scales) -> None:
        assert k_codes.dim() == 5 and k_codes.shape[3] == 32 and k_scales.dim() == 3 and v_codes.dim() == 8
        pages, heads, blocks, _, dim = k_codes.shape
        assert tuple(v_codes.shape) == (pages, heads, blocks, dim // 32, 16, 4, 2, 8) and tuple(k_scales.shape) == tuple(v_scales.shape) == (pages, heads, blocks)
        for t in (k_codes, k_scales, v_codes, v_scales):
            assert t.dtype == torch.uint8 and t.is_cuda and t.is_contiguous()
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.pages, self.kv_heads, self.head_dim, self.page_tokens, self.device = pages, heads, dim, 32 * blocks, k_codes.device
        self.shape = S.KVShape(heads, dim, self.page_tokens)
        self.cdesc = S.KVCacheDev(k_codes.data_ptr(), v_codes.data_ptr(), k_scales.data_ptr(), v_scales.data_ptr(), pages, self.shape)

    def _rows(self, t, heads: Optional[int], tokens: int, name: str):
        shape = t.shape
        assert len(shape) == 3 and shape[0] == tokens and shape[2] == self.head_dim and (heads is None or shape[1] == heads), f"{name}: shape {tuple(shape)}"
        token, head, channel = t.stride()
        assert t.dtype is torch.bfloat16 and t.is_cuda and channel == 1, f"{name}: bf16 [tokens, heads, head_dim] on the GPU, channels next to each other"
        return S.KVRowsDev(t.data_ptr(), token, head)

    def _stream(self, stream):
        return _current_stream(self.device.index) if stream is None else stream.cuda_stream

    def _new(self, shape, dtype, stream):
        """Memory for a call on `stream`.  It is that stream's (what the current one still does with memory that it gave back does not reach it), and the caller's on the
        current one: not given out again before both are done with it."""
        if stream is None:
            return torch.empty(shape, dtype=dtype, device=self.device)
        current = torch.cuda.current_stream(self.device)
        with torch.cuda.stream(stream):
            t = torch.empty(shape, dtype=dtype, device=self.device)
        if current != stream:
            t.record_stream(current)
        return t

    def append(self, k, v, batch: KVBatch, rope: Optional[Rope] = None, stream=None) -> None:
        """k, v: bf16 [new_tokens, kv_heads, head_dim] (any token and head stride that keeps 16-byte alignment)."""
        kd, vd = self._rows(k, self.kv_heads, batch.new_tokens, "k"), self._rows(v, self.kv_heads, batch.new_tokens, "v")
        S._check(S.lib().svdq_kv_append(self.cdesc, batch.cdesc, None if rope is None else rope.cdesc, kd, vd, self._stream(stream)), "svdq_kv_append")

    def attention_workspace(self, batch: KVBatch, q_heads: int, stream=None):
        n = S.lib().svdq_kv_attention_workspace_bytes(C.byref(self.shape), int(q_heads), batch.sequences, batch.max_new, batch.max_len)
        if n == 0:
            raise S.SvdqError("unsupported shape")
        return self._new(n, torch.uint8, stream)

    def attention(self, q, batch: KVBatch, rope: Optional[Rope] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                  out=None, workspace=None, stream=None):
        """q: bf16 [new_tokens, q_heads, head_dim].  Returns bf16 of the same shape, contiguous.  scale: 1 / sqrt(head_dim) if None."""
        qd = self._rows(q, None, batch.new_tokens, "q")
        heads = q.shape[1]
        if out is None:
            out = self._new((batch.new_tokens, heads, self.head_dim), torch.bfloat16, stream)
        else:
            assert out.dtype is torch.bfloat16 and out.is_cuda and out.is_contiguous() and out.shape == q.shape
        if workspace is None:
            workspace = self.attention_workspace(batch, heads, stream)
        else:
            assert workspace.dtype is torch.uint8 and workspace.is_cuda and workspace.is_contiguous(), "workspace: uint8 on the GPU"
        S._check(S.lib().svdq_kv_attention(self.cdesc, batch.cdesc, None if rope is None else rope.cdesc, qd, heads,
                                           1.0 / math.sqrt(self.head_dim) if scale is None else float(scale), int(causal), int(window), out.data_ptr(),
                                           workspace.data_ptr(), workspace.numel(), self._stream(stream)), "svdq_kv_attention")
        return out

    def gather(self, rows: KVRows, out=None, stream=None):
        """Keys and values bf16 [rows, kv_heads, head_dim] as they are held."""
        shape = (rows.rows, self.kv_heads, self.head_dim)
        if out is None:
            out = [self._new(shape, torch.bfloat16, stream) for _ in range(2)]
        for t in out:
            assert t.dtype is torch.bfloat16 and t.is_cuda and t.is_contiguous() and t.shape == shape
        S._check(S.lib().svdq_kv_gather(self.cdesc, *rows.pointers, rows.sequences, rows.width, rows.rows, out[0].data_ptr(), out[1].data_ptr(), self._stream(stream)),
                 "svdq_kv_gather")
        return out
