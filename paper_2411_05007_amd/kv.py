"""Binding of the paged 8-bit cache of keys and values, of the attention over it and of its pages (``svdq_kv_*`` in ``include/svdq.h``).

    cache = KVCache(pages, kv_heads, head_dim, page_tokens)
    batch = KVBatch(cu_new, kv_len, block_table, new_tokens, max_new, max_len)
    q, k, v = split_heads(qkv, q_heads, kv_heads)                     # views of a QKV layer's output
    cache.append(k, v, batch, rope)                                   # keys rotated, both quantized
    out = cache.attention(q, batch, rope)                             # bf16 [tokens, q_heads, head_dim]

A stream that outlives its window, in pages that are handed out and given back on the GPU:

    norm, pool = KVNorm(q_weight, k_weight), KVPages(pages, page_tokens)
    pool.reserve(cache, batch)                                        # the new tokens' pages
    cache.append(k, v, batch, rope, norm=norm)
    out = cache.attention(q, batch, rope, window=4096, sinks=4, norm=norm)
    pool.release(batch.block_table, first_token, end_token)           # what lies between the first tokens and the window
    cache.compact(moves, rope)                                        # or: some tokens become a sequence's only ones

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


class KVNorm:
    """Norm of queries and keys for each head, before the rotation: w x / sqrt(mean x^2 + eps).  q, k: fp32 weights on the GPU, [head_dim] or [heads, head_dim] (both alike);
    None: ones.  Tokens at positions below first_tokens take q_first and k_first."""

    def __init__(self, q=None, k=None, eps: float = 1e-6, q_first=None, k_first=None, first_tokens: int = 0):
        self.q, self.k, self.q_first, self.k_first, self.eps = q, k, q_first, k_first, float(eps)
        given = [t for t in (q, k, q_first, k_first) if t is not None]
        for t in given:
            assert t.dtype is torch.float32 and t.is_cuda and t.is_contiguous() and t.dim() in (1, 2), "weights: contiguous fp32 [head_dim] or [heads, head_dim] on the GPU"
        assert len({(t.dim(), t.shape[-1]) for t in given}) <= 1, "weights: all for each head, or none, and of one head size"
        for a, b in ((q, q_first), (k, k_first)):
            assert a is None or b is None or a.shape == b.shape, "weights: of the first tokens as of the others"
        heads = lambda a, b: next((t.shape[0] for t in (a, b) if t is not None and t.dim() == 2), None)
        self.q_heads, self.k_heads, self.dim = heads(q, q_first), heads(k, k_first), given[0].shape[-1] if given else None      # (None: any)
        at = lambda t: None if t is None else t.data_ptr()
        self.cdesc = S.KVNormDev(at(q), at(k), at(q_first), at(k_first), int(first_tokens), int(bool(given) and given[0].dim() == 2), self.eps)

    def _check(self, held: Optional[int], heads: int, dim: int) -> None:
        assert (self.dim is None or self.dim == dim) and (held is None or held == heads), f"norm: weights of {self.dim} channels and {held} heads for {heads} heads of {dim}"


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


class KVMoves:
    """Tokens that become a sequence's tokens from to_first[b] on: those of numbers from_token[cu_moves[b]] .. from_token[cu_moves[b + 1] - 1], in that order.  All int32 on the
    GPU: cu_moves [B + 1], from_token [moves] or [1, moves], or [kv_heads, moves] for lists of each head's own, to_first [B], from_table and to_table [B, width]."""

    def __init__(self, cu_moves, from_token, to_first, from_table, to_table, moves: int):
        for t, n in ((cu_moves, "cu_moves"), (from_token, "from_token"), (to_first, "to_first"), (from_table, "from_table"), (to_table, "to_table")):
            _device_int32(t, n)
        B = to_first.shape[0]
        assert cu_moves.shape == (B + 1,) and from_table.dim() == 2 and to_table.dim() == 2 and from_table.shape[0] == to_table.shape[0] == B
        assert from_token.dim() in (1, 2) and from_token.shape[-1] == moves, "from_token: [moves] or [heads, moves]"
        self.cu_moves, self.from_token, self.to_first, self.from_table, self.to_table, self.sequences, self.moves = cu_moves, from_token, to_first, from_table, to_table, B, int(moves)
        self.lists = 1 if from_token.dim() == 1 else from_token.shape[0]
        self.cdesc = S.KVMovesDev(cu_moves.data_ptr(), from_token.data_ptr(), to_first.data_ptr(), from_table.data_ptr(), to_table.data_ptr(), B, from_table.shape[1],
                                  to_table.shape[1], self.moves, int(self.lists > 1))


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

    def append(self, k, v, batch: KVBatch, rope: Optional[Rope] = None, stream=None, norm: Optional[KVNorm] = None) -> None:
        """k, v: bf16 [new_tokens, kv_heads, head_dim] (any token and head stride that keeps 16-byte alignment)."""
        kd, vd = self._rows(k, self.kv_heads, batch.new_tokens, "k"), self._rows(v, self.kv_heads, batch.new_tokens, "v")
        if norm is not None:
            norm._check(norm.k_heads, self.kv_heads, self.head_dim)
        S._check(S.lib().svdq_kv_append_normed(self.cdesc, batch.cdesc, None if norm is None else norm.cdesc, None if rope is None else rope.cdesc, kd, vd,
                                               self._stream(stream)), "svdq_kv_append")

    def attention_workspace(self, batch: KVBatch, q_heads: int, stream=None):
        n = S.lib().svdq_kv_attention_workspace_bytes(C.byref(self.shape), int(q_heads), batch.sequences, batch.max_new, batch.max_len)
        if n == 0:
            raise S.SvdqError("unsupported shape")
        return self._new(n, torch.uint8, stream)

    def attention(self, q, batch: KVBatch, rope: Optional[Rope] = None, scale: Optional[float] = None, causal: bool = True, window: int = 0,
                  out=None, workspace=None, stream=None, norm: Optional[KVNorm] = None, sinks: int = 0):
        """q: bf16 [new_tokens, q_heads, head_dim].  Returns bf16 of the same shape, contiguous.  scale: 1 / sqrt(head_dim) if None.  window: how many of the last tokens a
        row sees (0: all), sinks: first tokens of a sequence that it sees beside them."""
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
        if norm is not None:
            norm._check(norm.q_heads, heads, self.head_dim)
        S._check(S.lib().svdq_kv_attention_normed(self.cdesc, batch.cdesc, None if norm is None else norm.cdesc, None if rope is None else rope.cdesc, qd, heads,
                                                  1.0 / math.sqrt(self.head_dim) if scale is None else float(scale), int(causal), int(window), int(sinks), out.data_ptr(),
                                                  workspace.data_ptr(), workspace.numel(), self._stream(stream)), "svdq_kv_attention")
        return out

    def copy_pages(self, copies, source: Optional["KVCache"] = None, stream=None) -> None:
        """copies int32 [n, 3] on the GPU: page of `source` (None: of this cache), page of this cache, tokens (whole blocks of 32 are copied; rows that name no page are skipped).
        No other row of a table names a page that is written."""
        _device_int32(copies, "copies")
        assert copies.dim() == 2 and copies.shape[1] == 3, "copies: [n, 3]"
        S._check(S.lib().svdq_kv_copy_pages(self.cdesc, (source or self).cdesc, copies.data_ptr(), copies.shape[0], self._stream(stream)), "svdq_kv_copy_pages")

    def compact_workspace(self, moves: KVMoves, stream=None):
        n = S.lib().svdq_kv_compact_workspace_bytes(C.byref(self.shape), moves.sequences, moves.moves)
        if n == 0:
            raise S.SvdqError("unsupported shape")
        return self._new(n, torch.uint8, stream)

    def compact(self, moves: KVMoves, rope: Optional[Rope] = None, source: Optional["KVCache"] = None, workspace=None, stream=None) -> None:
        """Moves tokens into pages of this cache, out of pages of `source` (None: of this cache).  rope: turns their keys to the new positions.  workspace (compact_workspace()):
        needed where pages that are written are read as well.  Pages that are written are named by no other row: a branch whose pages others share is compacted into a row of its own,
        which reserve() fills, and its old row is released."""
        assert moves.lists in (1, self.kv_heads), f"from_token: {moves.lists} lists for {self.kv_heads} heads"
        assert workspace is None or (workspace.dtype is torch.uint8 and workspace.is_cuda and workspace.is_contiguous()), "workspace: uint8 on the GPU"
        at, size = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.numel())
        S._check(S.lib().svdq_kv_compact(self.cdesc, (source or self).cdesc, moves.cdesc, None if rope is None else rope.cdesc, at, size, self._stream(stream)), "svdq_kv_compact")

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


class KVPages:
    """Which pages are in use, by how many table entries, on the GPU: tables whose rows share pages are changed by fork(), reserve() and release() alone.

        pool = KVPages(pages, page_tokens)                   # one for the caches of all layers
        pool.fork(table, kv_len, parent, branch_table, branch_len)      # branches share the pages of their parents
        pool.reserve(cache, batch)                           # before append(): the new tokens' pages exist and are the sequence's own
        pool.release(branch_table)                           # given back
    """

    def __init__(self, pages: int, page_tokens: int = 64, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise S.SvdqError("no GPU visible: the pages have no CPU path")
        self._own(torch.zeros(pages, dtype=torch.int32, device=device), page_tokens)

    @classmethod
    def from_counts(cls, refs, page_tokens: int = 64) -> "KVPages":
        """Over counts int32 [pages] that are there already; they are kept, not copied."""
        self = cls.__new__(cls)
        self._own(refs, page_tokens)
        return self

    def _own(self, refs, page_tokens: int) -> None:
        _device_int32(refs, "refs")
        assert refs.dim() == 1
        self.refs, self.pages, self.page_tokens, self.device = refs, refs.shape[0], int(page_tokens), refs.device
        self.cdesc = S.KVPoolDev(refs.data_ptr(), self.pages, self.page_tokens)

    _stream, _new = KVCache._stream, KVCache._new

    @staticmethod
    def _table(t, name: str):
        assert t.dtype is torch.int32 and t.is_cuda and t.is_contiguous() and t.dim() == 2, f"{name}: contiguous int32 [sequences, width] on the GPU"
        return t.shape

    @staticmethod
    def _one_each(t, rows: int, name: str) -> int:
        assert t.dtype is torch.int32 and t.is_cuda and t.is_contiguous() and t.dim() == 1 and t.numel() == rows, f"{name}: contiguous int32 on the GPU, one for each row"
        return t.data_ptr()

    def release(self, block_table, first_token=None, end_token=None, stream=None) -> None:
        """Gives back the pages wholly within tokens first_token[b] .. end_token[b] - 1 of each row (None: from 0, to the end); the entries become -1."""
        rows, width = self._table(block_table, "block_table")
        first = None if first_token is None else self._one_each(first_token, rows, "first_token")
        end = None if end_token is None else self._one_each(end_token, rows, "end_token")
        S._check(S.lib().svdq_kv_pages_release(self.cdesc, block_table.data_ptr(), first, end, rows, width, self._stream(stream)), "svdq_kv_pages_release")

    def fork(self, from_table, from_len, parent, to_table, to_len, stream=None) -> None:
        """Rows of to_table take the pages of rows parent[i] of from_table, to_len[i] becomes from_len[parent[i]].  What to_table named before is to be released first."""
        parents, from_width = self._table(from_table, "from_table")
        rows, to_width = self._table(to_table, "to_table")
        S._check(S.lib().svdq_kv_pages_fork(self.cdesc, from_table.data_ptr(), self._one_each(from_len, parents, "from_len"), parents, from_width,
                                            self._one_each(parent, rows, "parent"), to_table.data_ptr(), self._one_each(to_len, rows, "to_len"), rows, to_width,
                                            self._stream(stream)), "svdq_kv_pages_fork")

    def reserve_workspace(self, batch: KVBatch, stream=None):
        """For reserve(): its notes, and what further caches copy."""
        return self._new(self._notes(batch) + 12 * batch.sequences, torch.uint8, stream)

    def _notes(self, batch: KVBatch) -> int:
        n = S.lib().svdq_kv_pages_reserve_workspace_bytes(C.byref(self.cdesc), batch.sequences, batch.block_table.shape[1])
        if n == 0:
            raise S.SvdqError("unsupported pool")
        return n

    def reserve(self, cache, batch: KVBatch, missing=None, workspace=None, stream=None) -> None:
        """Pages of its own for every new token of the batch, whose block_table is written; tokens before them in a shared page are copied, in `cache` or, where layers
        have caches of their own, in each of a list of them (in none of an empty list).  missing: int32 [1] on the GPU, entries for which no page was left (they name none), and those that cannot have
        one: a sequence's first that names none while tokens before the new ones fall in it.  Written anew by each call: a captured step adds it up in a tensor of its own."""
        caches = [cache] if isinstance(cache, KVCache) else list(cache)
        for c in caches:
            assert c.pages >= self.pages and c.page_tokens == self.page_tokens, f"cache: {c.pages} pages of {c.page_tokens} for a pool of {self.pages} of {self.page_tokens}"
        if missing is not None:
            _device_int32(missing, "missing")
            assert missing.numel() == 1
        if workspace is None:
            workspace = self.reserve_workspace(batch, stream)
        else:
            assert workspace.dtype is torch.uint8 and workspace.is_cuda and workspace.is_contiguous(), "workspace: uint8 on the GPU"
        L, at, size, copies = S.lib(), workspace.data_ptr(), workspace.numel(), None
        if len(caches) > 1:
            size = self._notes(batch)
            if workspace.numel() < size + 12 * batch.sequences:
                raise S.SvdqError("svdq_kv_pages_reserve: workspace smaller than reserve_workspace()")
            copies = at + size
        s = self._stream(stream)
        S._check(L.svdq_kv_pages_reserve(self.cdesc, caches[0].cdesc if caches else None, batch.cdesc, copies, None if missing is None else missing.data_ptr(), at, size, s),
                 "svdq_kv_pages_reserve")
        for c in caches[1:]:
            S._check(L.svdq_kv_copy_pages(c.cdesc, c.cdesc, copies, batch.sequences, s), "svdq_kv_copy_pages")
