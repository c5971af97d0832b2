"""Workloads of the operators between a block's QKV layer and its output layer: the paged 8-bit cache of keys and values.

  append     rotates the keys of new tokens by their positions, quantizes keys and values to E4M3 codes with a power-of-two
             scale byte for each 32 tokens and head, and writes them into the pages of a cache
  attention  softmax(scale q k^T) v of the new tokens over that cache, with the queries rotated on the way in
  gather     reads rows of the cache back as 16-bit values

The format.  A cache has pages of P tokens, cut into blocks of 32.  Keys: uint8 [pages][heads][P / 32][32][D], E4M3 codes.
Values: uint8 [pages][heads][P / 32][D / 32][16][4][2][8], transposed: element (t, d) of a block lies at
[d / 32][d % 16][2 (t / 16) + (t % 8) / 4][(d % 32) / 16][4 ((t % 16) / 8) + t % 4].  Scale bytes: uint8 [pages][heads][P / 32]
for each of the two; a code c of a block with byte b stands for c * 2^(b - 127), byte 0 marks a block of zeros.
The byte of a block is that of the smallest power of two s >= 2^-126 with max|x| <= 448 s; while a block fills, its byte only
grows and the codes that are in it already are rounded again.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"


def _kv():
    from paper_2411_05007_amd import kv
    return kv


# ---------------------------------------------------------------------------------------------------------------------
# cases


def _case(name, kind, B, q_heads, kv_heads, D, new, before, page=64, causal=True, window=0, rot=None, interleaved=False, mix=0):
    """new, before: (least, most) new tokens of a sequence and tokens that its cache holds already; the first sequence has the most of both."""
    c = {"kind": kind, "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "new_lo": new[0], "new_hi": new[1], "before_lo": before[0],
         "before_hi": before[1], "page": page, "causal": causal, "window": window, "rot": D if rot is None else rot, "interleaved": interleaved, "mix": mix}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one token for each sequence of a serving batch
        _case("append_step_64", "append", 64, 32, 8, 128, (1, 1), (200, 8191)),
        # ragged prompts behind cached prefixes, narrow heads, odd lengths, rotation of a part of the channels
        _case("append_ragged_d64", "append", 7, 12, 12, 64, (3, 1777), (0, 501), page=32, rot=32),
        # keys and values of the 24 heads of a FLUX.1 block (3072 = 24 * 128), four images of 4608 tokens; its rotation takes neighbouring channels
        _case("append_joint_4x4608", "append", 4, 24, 24, 128, (4608, 4608), (0, 0), page=128, interleaved=True),
        # the smallest call: one sequence, one token, a short context
        _case("attention_step_1x777", "attention", 1, 32, 8, 128, (1, 1), (776, 776)),
        # one sequence, one token, a long context
        _case("attention_step_1x131071", "attention", 1, 32, 8, 128, (1, 1), (131070, 131070), page=256),
        # a serving batch with contexts of all lengths
        _case("attention_step_64x16k", "attention", 64, 32, 8, 128, (1, 1), (100, 16383)),
        # every head its own keys, narrow heads, up to five tokens in a step, a sliding window
        _case("attention_few_d64_window", "attention", 24, 16, 16, 64, (1, 5), (37, 6001), page=32, window=1024, rot=32),
        # ragged prompts behind cached prefixes
        _case("attention_chunks_ragged", "attention", 6, 32, 8, 128, (17, 2111), (0, 1500), mix=3),
        # joint attention of the 4608 text and image tokens of a FLUX.1 block, 24 heads, every token sees every other
        _case("attention_joint_4608", "attention", 1, 24, 24, 128, (4608, 4608), (0, 0), page=128, causal=False, interleaved=True),
        # a chunk of a long prompt: the largest pass
        _case("attention_chunk_8k_of_16k", "attention", 1, 32, 8, 128, (8192, 8192), (8192, 8192), page=128),
        # a shared prefix, and the prefixes of a batch, as 16-bit rows
        _case("gather_prefix_1x1000", "gather", 1, 32, 8, 128, (1, 1), (999, 999)),
        _case("gather_prefix_16x4k", "gather", 16, 32, 8, 128, (1, 1), (50, 4095), page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what a drawn case may not exceed: scores (heads * new tokens * keys, padded to the longest sequence) of the largest listed pass, tokens held in all
MAX_SCORES = 32 * 8192 * 16384
MAX_ELEMENTS = 64 * 16384 * 8 * 128


def draw(rng):
    kind = rng.choice(["append", "step", "step", "few", "chunk", "chunk", "joint", "gather"])
    D = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 24])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 8] if kv_heads <= 8 else [1, 2])
    page = rng.choice([32, 64, 128, 256])
    rot = rng.choice([D, D, D // 2])
    B = _log_int(rng, 1, 64)
    before = _log_int(rng, 1, 131072 if kind == "step" else 16384) - (rng.random() < 0.2)
    new = {"append": _log_int(rng, 1, 8192), "step": 1, "few": rng.randint(2, 8), "chunk": _log_int(rng, 9, 8192), "joint": _log_int(rng, 16, 8192),
           "gather": 1}[kind]
    if kind == "joint":
        before = 0
    while B > 1 and (B * q_heads * new * (before + new) > MAX_SCORES or B * (before + new) * kv_heads * D > MAX_ELEMENTS):
        B = B // 2
    if q_heads * new * (before + new) > MAX_SCORES:
        before = max(0, MAX_SCORES // (q_heads * new) - new)
        new = min(new, int(math.sqrt(MAX_SCORES / q_heads)))
    if (before + new) * kv_heads * D > MAX_ELEMENTS:
        before = max(0, MAX_ELEMENTS // (kv_heads * D) - new)
    window = _log_int(rng, 16, 4096) if kind in ("step", "few", "chunk") and rng.random() < 0.25 else 0
    return _case(None, kind if kind in ("append", "gather") else "attention", B, q_heads, kv_heads, D, (max(1, new // 20), new), (before // 20, before), page,
                 kind != "joint", window, rot, rng.random() < 0.3, rng.randint(0, 999))


def _lengths(case):
    """[(tokens held before, new tokens)] of the sequences."""
    rng = random.Random(case["mix"] * 1000003 + case["B"])
    got = [(case["before_hi"], case["new_hi"])]
    for _ in range(case["B"] - 1):
        got.append((rng.randint(case["before_lo"], case["before_hi"]), rng.randint(case["new_lo"], case["new_hi"])))
    return got


# ---------------------------------------------------------------------------------------------------------------------
# inputs


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _scale_byte(amax):
    """Byte of the smallest power of two s >= 2^-126 with amax <= 448 s (0 for amax = 0), from the bits of an fp32 maximum."""
    bits = amax.contiguous().view(torch.int32)
    byte = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 254)
    return torch.where(amax > 0, byte, torch.zeros_like(byte))


def _pow2(e):
    """2^e in fp32 for integer e; 0 below the smallest normal number."""
    return torch.where(e < -126, torch.zeros_like(e), (e.clamp(-126, 127) + 127) << 23).int().view(torch.float32)


def _e4m3(x):
    """Codes (uint8) of the E4M3 numbers nearest to x, |x| <= 448."""
    return x.to(torch.float8_e4m3fn).view(torch.uint8)


def _values_in_order(v):
    """[..., 32 tokens, D] of a block to the order of the cache, [..., D / 32, 16, 4, 2, 8]."""
    lead, D, n = v.shape[:-2], v.shape[-1], v.dim() - 2
    v = v.reshape(*lead, 2, 2, 2, 4, D // 32, 2, 16)      # [token / 16][(token % 16) / 8][(token % 8) / 4][token % 4][d / 32][(d % 32) / 16][d % 16]
    v = v.permute(*range(n), n + 4, n + 6, n, n + 2, n + 5, n + 1, n + 3)
    return v.reshape(*lead, D // 32, 16, 4, 2, 8)


def _values_by_token(v):
    """The way back: [..., D / 32, 16, 4, 2, 8] to [..., 32, D]."""
    lead, A, n = v.shape[:-5], v.shape[-5], v.dim() - 5
    v = v.reshape(*lead, A, 16, 2, 2, 2, 2, 4)            # [d / 32][d % 16][token / 16][(token % 8) / 4][(d % 32) / 16][(token % 16) / 8][token % 4]
    v = v.permute(*range(n), n + 2, n + 5, n + 3, n + 6, n, n + 4, n + 1)
    return v.reshape(*lead, 32, A * 32)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    B, Hq, Hkv, D, P = case["B"], case["q_heads"], case["kv_heads"], case["D"], case["page"]
    lengths = _lengths(case)
    width = max((b + n + P - 1) // P for b, n in lengths)
    need = [(b + n + P - 1) // P for b, n in lengths]
    pages = sum(need) + 2
    # the pages of a sequence lie anywhere in the cache
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    table = torch.zeros(B, width, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    # keys have a few channels that are larger; blocks differ in scale
    loud = 1.0 + 3.0 * (torch.rand(Hkv, 1, 1, D, generator=gen, device=DEV) < 0.02).float()

    def filled(gain):
        codes = torch.empty(pages, Hkv, P // 32, 32, D, dtype=torch.uint8, device=DEV)
        scales = torch.empty(pages, Hkv, P // 32, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 28) // (Hkv * P * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = _normal(gen, n, Hkv, P // 32, 32, D) * gain * torch.exp2(torch.rand(n, Hkv, P // 32, 1, 1, generator=gen, device=DEV) - 0.5)
            byte = _scale_byte(x.abs().amax(dim=(-1, -2)))
            codes[p:p + n] = _e4m3(x * _pow2(127 - byte)[..., None, None])
            scales[p:p + n] = byte.to(torch.uint8)
        return codes, scales

    k_codes, k_scales = filled(loud)
    v_codes, v_scales = filled(1.0)
    v_codes = _values_in_order(v_codes).contiguous()
    new = [n for _, n in lengths]
    T = sum(new)
    # what the QKV layer leaves: one row a token, queries, keys and values of all heads behind each other
    qkv = _normal(gen, T, (Hq + 2 * Hkv), D)
    qkv[:, Hq:Hq + Hkv] *= loud.view(Hkv, D)
    qkv = qkv.to(torch.bfloat16)
    # rotation by position, angles p * 10000^(-2 i / r)
    r = case["rot"]
    most = max(b + n for b, n in lengths)
    angle = torch.arange(most, device=DEV, dtype=torch.float64)[:, None] * torch.exp2(-math.log2(10000.0) * 2.0 / r * torch.arange(r // 2, device=DEV, dtype=torch.float64))
    rope = torch.cat([angle.cos(), angle.sin()], dim=1).float().contiguous()
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    # rows that are read back: an append's from the first block that it touches, a gather's from a few tokens in
    start = [b // 32 * 32 if case["kind"] == "append" else min(5, b) for b, _ in lengths]
    cu_rows = [0]
    for (b, n), s in zip(lengths, start):
        cu_rows.append(cu_rows[-1] + b + n - s)
    return {"case": dict(case), "k_codes": k_codes, "k_scales": k_scales, "v_codes": v_codes, "v_scales": v_scales, "qkv": qkv, "rope": rope, "table": table,
            "cu": _i32(cu), "kv_len": _i32([b + n for b, n in lengths]), "start": _i32(start), "cu_rows": _i32(cu_rows), "rows": cu_rows[-1], "T": T,
            "max_new": max(new), "max_len": most,
            "out": torch.empty(T, Hq, D, dtype=torch.bfloat16, device=DEV) if case["kind"] == "attention" else None,
            "rows_out": [torch.empty(cu_rows[-1], Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)] if case["kind"] != "attention" else None}


# ---------------------------------------------------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c = s["case"]
    if "cache" not in s:      # a program keeps these
        KV = _kv()
        s["cache"] = KV.KVCache.from_buffers(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
        s["batch"] = KV.KVBatch(s["cu"], s["kv_len"], s["table"], s["T"], s["max_new"], s["max_len"])
        s["rotation"] = KV.Rope(s["rope"], interleaved=c["interleaved"])
        s["rows_batch"] = KV.KVRows(s["start"], s["cu_rows"], s["table"], s["rows"])
        s["workspace"] = s["cache"].attention_workspace(s["batch"], c["q_heads"]) if c["kind"] == "attention" else None
    Hq, Hkv = c["q_heads"], c["kv_heads"]
    if c["kind"] == "attention":
        return s["cache"].attention(s["qkv"][:, :Hq], s["batch"], rope=s["rotation"], causal=c["causal"], window=c["window"], out=s["out"], workspace=s["workspace"])
    if c["kind"] == "append":
        s["cache"].append(s["qkv"][:, Hq:Hq + Hkv], s["qkv"][:, Hq + Hkv:], s["batch"], rope=s["rotation"])
    return s["cache"].gather(s["rows_batch"], out=s["rows_out"])


def _rotate(x, position, rope, interleaved):
    r = rope.shape[1]
    c, s = rope[position, : r // 2][:, None, :], rope[position, r // 2:][:, None, :]
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _token_places(s):
    """sequence and position of every new token"""
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(new.numel(), device=DEV), new, output_size=s["T"])
    return b, torch.arange(s["T"], device=DEV) - s["cu"].long()[b] + (s["kv_len"].long() - new)[b]


def _from_codes(codes, byte):
    return codes.view(torch.float8_e4m3fn).float() * _pow2(byte.int() - 127)[..., None, None]


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "attention":
        return _attention_plain(s)
    if c["kind"] == "append":
        _append_plain(s)
    # rows read back
    n = (s["cu_rows"][1:] - s["cu_rows"][:-1]).long()
    b = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=s["rows"])
    t = torch.arange(s["rows"], device=DEV) - s["cu_rows"].long()[b] + s["start"].long()[b]
    page, block, at = s["table"].long()[b, t // c["page"]], t % c["page"] // 32, t % 32
    k = s["k_codes"].view(torch.float8_e4m3fn)[page, :, block, at].float() * _pow2(s["k_scales"][page, :, block].int() - 127)[..., None]
    v = s["v_codes"][page, :, block, :, :, 2 * (at // 16) + at % 8 // 4, :, 4 * (at % 16 // 8) + at % 4]      # [rows][head][D / 32][16][2]
    v = v.transpose(-1, -2).reshape(k.shape).contiguous().view(torch.float8_e4m3fn).float() * _pow2(s["v_scales"][page, :, block].int() - 127)[..., None]
    s["rows_out"][0].copy_(k)
    s["rows_out"][1].copy_(v)
    return s["rows_out"]


def _append_plain(s):
    c = s["case"]
    Hq, Hkv, D, P = c["q_heads"], c["kv_heads"], c["D"], c["page"]
    b, t = _token_places(s)
    k = _rotate(s["qkv"][:, Hq:Hq + Hkv].float(), t, s["rope"], c["interleaved"])
    v = s["qkv"][:, Hq + Hkv:].float()
    page, block, at = s["table"].long()[b, t // P], t % P // 32, t % 32
    blocks = P // 32
    # the block that a sequence's first new token falls in may hold tokens already; all others are new
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    first = s["kv_len"].long() - new
    some = (first % 32 > 0) & (new > 0)
    page0, block0 = s["table"].long().gather(1, (first // P).clamp(max=s["table"].shape[1] - 1)[:, None])[:, 0], first % P // 32
    held = torch.zeros(s["k_scales"].shape[0], blocks, dtype=torch.bool, device=DEV)
    held[page0[some], block0[some]] = True
    bad = ~(torch.isfinite(k).all(-1) & torch.isfinite(v).all(-1))
    for x, codes, scales, empty in ((k, s["k_codes"], s["k_scales"], float("nan")), (v, s["v_codes"], s["v_scales"], 0.0)):
        amax = torch.where(bad, torch.zeros((), device=DEV), x.abs().amax(-1))
        top = torch.zeros(scales.shape[0] * blocks, Hkv, device=DEV).index_reduce_(0, page * blocks + block, amax, "amax")
        byte = _scale_byte(top)[page * blocks + block]                                       # [token][head]
        old = torch.where(held[page, block][:, None], scales[page, :, block].int(), 0)
        byte = torch.maximum(byte, old)
        was = scales[page0, :, block0].int()                                                 # of the first blocks, before
        scales[page, :, block] = byte.to(torch.uint8)
        # what the first blocks hold, at the scale that they have now
        now = scales[page0, :, block0].int()
        kept = codes[page0, :, block0]                                                       # [sequence][head]...
        again = _e4m3(kept.view(torch.float8_e4m3fn).float() * _pow2((was - now).clamp(min=-100)).view(*was.shape, *[1] * (kept.dim() - 2)))
        again = torch.where((some[:, None] & (now > was)).view(*was.shape, *[1] * (kept.dim() - 2)), again, kept)
        codes[page0, :, block0] = again
        fresh = _e4m3(torch.where(bad[..., None], empty, x * _pow2(127 - byte)[..., None]))
        if codes is s["k_codes"]:
            codes[page, :, block, at] = fresh
        else:
            codes[page, :, block, :, :, 2 * (at // 16) + at % 8 // 4, :, 4 * (at % 16 // 8) + at % 4] = fresh.view(*fresh.shape[:2], D // 32, 2, 16).transpose(-1, -2)


def _attention_plain(s):
    c = s["case"]
    B, Hq, Hkv, D = c["B"], c["q_heads"], c["kv_heads"], c["D"]
    g, n, L = Hq // Hkv, s["max_new"], s["table"].shape[1] * c["page"]
    b, t = _token_places(s)
    q = torch.zeros(B, n, Hq, D, device=DEV)
    i = torch.arange(s["T"], device=DEV) - s["cu"].long()[b]
    q[b, i] = _rotate(s["qkv"][:, :Hq].float(), t, s["rope"], c["interleaved"])
    q = q.view(B, n, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B * Hkv, n * g, D) * (1.0 / math.sqrt(D))
    table = s["table"].long()
    k = _from_codes(s["k_codes"][table], s["k_scales"][table]).transpose(1, 2).reshape(B * Hkv, L, D)
    x = torch.matmul(q, k.transpose(1, 2)).view(B, Hkv, n, g, L)
    del k
    length = s["kv_len"].long()
    new = (s["cu"][1:] - s["cu"][:-1]).long()
    key = torch.arange(L, device=DEV)
    seen = key < length[:, None, None]
    if c["causal"]:
        p = (length - new)[:, None] + torch.arange(n, device=DEV)
        seen = seen & (key <= p[..., None])
        if c["window"]:
            seen = seen & (key > p[..., None] - c["window"])
    seen = seen.view(B, 1, -1, 1, L)
    x.masked_fill_(~seen, float("-inf"))
    x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    x.div_(x.sum(-1, keepdim=True).clamp(min=1e-30))
    v = _values_by_token(s["v_codes"][table])
    v = _from_codes(v, s["v_scales"][table]).transpose(1, 2).reshape(B, Hkv, L, D)
    v.masked_fill_((key >= length[:, None]).view(B, 1, L, 1), 0.0)
    o = torch.matmul(x.view(B * Hkv, n * g, L), v.view(B * Hkv, L, D))
    o = o.view(B, Hkv, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    s["out"].copy_(o[b, i])
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["D"]
    nbytes, flops = 0, 0
    for before, new in _lengths(case):
        L = before + new
        if case["kind"] == "attention":
            least, pairs = 0, new * L
            if case["causal"]:
                w = case["window"] or L
                pairs = sum(min(before + i + 1, w) for i in range(new))
                least = max(0, before + 1 - w)
            nbytes += 2 * (L - least) * Hkv * D + (L - least + 31) // 32 * Hkv * 2 + 4 * new * Hq * D + 4 * new * case["rot"]
            flops += 4 * D * Hq * pairs
        elif case["kind"] == "append":
            rows = L - before // 32 * 32
            nbytes += 4 * new * Hkv * D + 2 * new * Hkv * D + 4 * new * case["rot"] + 2 * rows * Hkv * D + 4 * rows * Hkv * D
            flops += 3 * new * Hkv * D
        else:
            rows = L - min(5, before)
            nbytes += 6 * rows * Hkv * D + (rows + 31) // 32 * Hkv * 2
            flops += 2 * rows * Hkv * D
    return {"bytes": nbytes, "flops": flops}


# ---------------------------------------------------------------------------------------------------------------------
# the definition in 64 bits, one sequence at a time


def _decode64(code):
    """The number that an E4M3 code stands for, from its bits."""
    c = code.long()
    sign, e, m = 1 - 2 * (c >> 7), (c >> 3) & 15, c & 7
    value = torch.where(e > 0, (8 + m).double() * torch.exp2((e - 10).double()), m.double() * 2.0 ** -9)
    return torch.where((c & 127) == 127, torch.full((), float("nan"), dtype=torch.float64, device=c.device), sign * value)


def _round64(x):
    """x rounded to the nearest E4M3 number, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _held64(s, b, tokens):
    """keys and values [heads][token][D] of the tokens of sequence b, and their scales' exponents"""
    c = s["case"]
    D, P, Hkv = c["D"], c["page"], c["kv_heads"]
    page, block, at = s["table"][b].long()[tokens // P], tokens % P // 32, tokens % 32
    head = torch.arange(Hkv, device=DEV)[:, None]
    unit = (page * Hkv + head) * (P // 32) + block                          # [head][token]
    d = torch.arange(D, device=DEV)
    k = s["k_codes"].view(-1)[unit[..., None] * (32 * D) + (at[:, None] * D + d)]
    slot, j = 2 * (at // 16) + at % 8 // 4, 4 * (at % 16 // 8) + at % 4
    v = s["v_codes"].view(-1)[unit[..., None] * (32 * D) + ((((d // 32) * 16 + d % 16) * 4 + slot[:, None]) * 2 + d % 32 // 16) * 8 + j[:, None]]
    ek, ev = s["k_scales"].view(-1)[unit].long() - 127, s["v_scales"].view(-1)[unit].long() - 127
    return _decode64(k), _decode64(v), ek, ev


def _turn64(x, position, s):
    """x [token][head][D] rotated in 64 bits"""
    r, y = s["rope"].shape[1], x.clone()
    for i in range(r // 2):
        one, two = (2 * i, 2 * i + 1) if s["case"]["interleaved"] else (i, i + r // 2)
        co, si = s["rope"][position, i].double()[:, None], s["rope"][position, r // 2 + i].double()[:, None]
        y[..., one] = x[..., one] * co - x[..., two] * si
        y[..., two] = x[..., two] * co + x[..., one] * si
    return y


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, D = case["q_heads"], case["kv_heads"], case["D"]
    out, at = [], 0
    rows = [[], []]
    for b, (before, new) in enumerate(_lengths(case)):
        L = before + new
        x = s["qkv"][at:at + new].double()
        at += new
        place = torch.arange(before, L, device=DEV)
        if case["kind"] == "attention":
            k, v, ek, ev = _held64(s, b, torch.arange(L, device=DEV))
            k, v = k * torch.exp2(ek.double())[..., None], v * torch.exp2(ev.double())[..., None]
            q = _turn64(x[:, :Hq], place, s)
            o = torch.zeros(new, Hq, D, dtype=torch.float64, device=DEV)
            step = max(1, (1 << 28) // L)
            for h in range(Hq):
                for i in range(0, new, step):
                    p = place[i:i + step]
                    score = q[i:i + step, h] @ k[h // (Hq // Hkv)].T / math.sqrt(D)
                    j = torch.arange(L, device=DEV)
                    if case["causal"]:
                        hidden = j > p[:, None]
                        if case["window"]:
                            hidden |= j <= p[:, None] - case["window"]
                        score.masked_fill_(hidden, float("-inf"))
                    o[i:i + step, h] = torch.softmax(score, dim=-1) @ v[h // (Hq // Hkv)]
            out.append(o)
            continue
        start = before // 32 * 32 if case["kind"] == "append" else min(5, before)
        if case["kind"] == "gather":
            k, v, ek, ev = _held64(s, b, torch.arange(start, L, device=DEV))
            rows[0].append((k * torch.exp2(ek.double())[..., None]).transpose(0, 1))
            rows[1].append((v * torch.exp2(ev.double())[..., None]).transpose(0, 1))
            continue
        held = before - start
        old = _held64(s, b, torch.arange(start, before, device=DEV)) if held else None
        for which, fresh in ((0, _turn64(x[:, Hq:Hq + Hkv], place, s)), (1, x[:, Hq + Hkv:])):
            fresh = fresh.transpose(0, 1)                                   # [head][token][D]
            span = (L - start + 31) // 32 * 32
            padded = torch.zeros(Hkv, span, D, dtype=torch.float64, device=DEV)
            padded[:, held:held + new] = fresh
            amax = padded.view(Hkv, -1, 32 * D).abs().amax(-1)
            e = torch.ceil(torch.log2((amax / 448).clamp(min=2.0 ** -126)))
            if held:
                e[:, 0] = torch.maximum(e[:, 0], old[2 + which][:, 0].double())
            e = e.repeat_interleave(32, dim=1)[..., None]
            got = _round64(padded * torch.exp2(-e))
            if held:
                got[:, :held] = _round64(old[which] * torch.exp2(old[2 + which].double()[..., None] - e[:, :held]))
            rows[which].append((got * torch.exp2(e))[:, :L - start].transpose(0, 1))
    if case["kind"] == "attention":
        return torch.cat(out)
    return [torch.cat(r) for r in rows]
