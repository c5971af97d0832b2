"""Workloads of what a long-running program does with the paged 8-bit cache of keys and values: streams that outlive their window, and branches of them.

  append   normalises the keys of new tokens for each head, rotates them by position, quantizes keys and values into the pages of a cache
  stream   attention of new tokens in a window, with the first tokens of a sequence visible to all; queries normalised and rotated on the way in
  branch   sequences take over the pages of others, and get pages of their own where they are about to write: counts and tables on the GPU
  compact  some of a sequence's tokens become its only ones: keys turned to their new positions, blocks quantized anew

The norm.  y = w x / sqrt(mean x^2 + eps) over the channels of a head, then the rotation: (a, b) -> (a cos - b sin, b cos + a sin).

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
EPS = 1e-6


def _kv():
    from paper_2411_05007_amd import kv
    return kv


# ---------------------------------------------------------------------------------------------------------------------
# cases


def _append(name, B, q_heads, kv_heads, D, new, before, page=64, rot=None, interleaved=False, per_head=False, first=0, mix=0):
    """new, before: (least, most) new tokens of a sequence and tokens that its cache holds already; the first sequence has the most of both."""
    c = {"kind": "append", "B": B, "q_heads": q_heads, "kv_heads": kv_heads, "D": D, "new_lo": new[0], "new_hi": new[1], "before_lo": before[0],
         "before_hi": before[1], "page": page, "rot": rot if rot is not None else D, "interleaved": interleaved, "per_head": per_head, "first": first, "mix": mix}
    return c if name is None else dict(c, name=name)


def _stream(name, B, q_heads, kv_heads, D, new, before, window, sinks, page=64, rot=None, interleaved=False, per_head=False, first=0, mix=0):
    return dict(_append(name, B, q_heads, kv_heads, D, new, before, page, rot, interleaved, per_head, first, mix), kind="stream", window=window, sinks=sinks)


def _branch(name, parents, children, kv_heads, D, new, before, page=64, spare=8, mix=0):
    """children of each parent; spare: pages that stay free, or (below zero) that lack."""
    c = {"kind": "branch", "B": parents, "children": children, "kv_heads": kv_heads, "D": D, "new_lo": new[0], "new_hi": new[1], "before_lo": before[0],
         "before_hi": before[1], "page": page, "spare": spare, "mix": mix}
    return c if name is None else dict(c, name=name)


def _compact(name, B, kv_heads, D, held, kept, choice, to=(0, 0), page=64, rot=0, interleaved=False, staged=False, mix=0):
    """held, kept: (least, most) tokens of a sequence and those of them that stay; choice: "recent" (the first few and the last), "tail" (some of the
    last 64), "some" (any) or "heads" (any, others for each head); to: (least, most) tokens before them; rot 0: keys stay as they are turned; staged: by way of a workspace."""
    c = {"kind": "compact", "B": B, "kv_heads": kv_heads, "D": D, "held_lo": held[0], "held_hi": held[1], "kept_lo": kept[0], "kept_hi": kept[1], "choice": choice,
         "to_lo": to[0], "to_hi": to[1], "page": page, "rot": rot, "interleaved": interleaved, "staged": staged, "mix": mix}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a step of 64 conversations: one token each
        _append("norm_append_64x1", 64, 32, 8, 128, (1, 1), (100, 8000)),
        # a guidance batch of joint blocks: 512 text tokens with weights of their own before 4096 image tokens
        _append("norm_append_joint_4x4608", 4, 24, 24, 128, (4608, 4608), (0, 0), page=128, interleaved=True, first=512),
        # ragged prompts behind cached prefixes, half of the head rotated, weights for each head
        _append("norm_append_ragged_d64", 6, 24, 12, 64, (17, 2111), (0, 1500), page=32, rot=32, per_head=True),
        # one long conversation, a token at a time: where latency counts
        _stream("stream_step_1x30k", 1, 32, 8, 128, (1, 1), (30000, 30000), 1024, 4),
        # 64 conversations of up to 32768 tokens in a window of 8192
        _stream("stream_step_64x32k", 64, 32, 8, 128, (1, 1), (100, 32767), 8192, 64, page=128, mix=1),
        # a few tokens each (a guess that is checked), three query heads on a key head of 64, odd lengths
        _stream("stream_few_d64", 24, 12, 4, 64, (1, 5), (0, 6001), 777, 33, page=32, rot=32, interleaved=True, per_head=True, mix=2),
        # a chunk of a long prompt
        _stream("stream_chunk_8k_of_24k", 1, 32, 8, 128, (8192, 8192), (16384, 16384), 8192, 128, page=128),
        # beam search and parallel sampling: four continuations of each prompt, a token each
        _branch("branch_8x4", 8, 4, 8, 128, (1, 1), (100, 2000)),
        # the same for many long prompts, pages of 256, some of them with a few tokens to check
        _branch("branch_64x4_p256", 64, 4, 4, 128, (1, 40), (1000, 8191), page=256, spare=64),
        # the accepted path of a tree of guesses: a few of the last tokens move together
        _compact("compact_tail_32x5", 32, 8, 128, (300, 2000), (1, 8), "tail", to=(200, 290), rot=128, staged=True),
        # the first tokens and the latest ones stay, other ones for each head
        _compact("compact_heads_16x4k", 16, 8, 128, (3000, 8192), (1000, 4096), "heads", page=128),
        # prompts thinned out, the keys turned to their new positions: the largest
        _compact("compact_some_64x12k", 64, 8, 128, (9000, 16384), (5000, 12001), "some", page=128, rot=128, mix=1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# what a drawn case may not exceed
MAX_SCORES = 32 * 8192 * 16384         # heads x new tokens x keys, padded
MAX_SEEN = 64 * 8192 * 8 * 128         # channels of the keys that are seen
MAX_CELLS = 64 * 16384 * 8 * 128       # channels of the keys that are held
MAX_NEW = 4 * 4608 * 24 * 128          # channels of new keys
MAX_PAGES = 1 << 28                    # codes of all pages of a branching pool (keys)


def draw(rng):
    kind = rng.choice(["append", "append", "step", "step", "few", "chunk", "branch", "branch", "compact", "compact", "compact"])
    D = rng.choice([64, 128, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 12, 24])
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 4, 8] if kv_heads <= 8 else [1, 2])
    page = rng.choice([32, 64, 128, 256])
    rot = rng.choice([D, D, D // 2])
    B = _log_int(rng, 1, 64)
    mix = rng.randint(0, 999)
    if kind == "branch":
        before, new, children = _log_int(rng, 1, 8191), rng.choice([1, 1, rng.randint(2, 64), _log_int(rng, 16, 700)]), rng.choice([1, 2, 3, 4, 8])
        pages = lambda: B * ((before + page - 1) // page + children * (2 + new // page)) * page * kv_heads * D
        while pages() > MAX_PAGES and B > 1:
            B //= 2
        while pages() > MAX_PAGES and before > 64:
            before //= 2
        return _branch(None, B, children, kv_heads, D, (1, new), (before // 10, before), page, rng.choice([-2, 0, 3, 50]), mix)
    if kind == "compact":
        held = _log_int(rng, 1, 16384)
        while B > 1 and B * held * kv_heads * D > MAX_CELLS:
            B //= 2
        held = max(1, min(held, MAX_CELLS // (kv_heads * D)))
        choice = rng.choice(["recent", "tail", "some", "heads"])
        kept = max(1, min(held, rng.randint(1, 20))) if choice == "tail" else max(1, int(held * rng.uniform(0.1, 1.0)))
        to = rng.choice([0, 0, rng.randint(1, 400)])
        return _compact(None, B, kv_heads, D, ((held + 1) // 2, held), ((kept + 1) // 2, kept), choice, (to // 2, to), page, rot if rng.random() < 0.6 else 0,
                        rng.random() < 0.3, rng.random() < 0.3, mix)
    before = _log_int(rng, 1, 100000 if kind == "step" else 16384) - (rng.random() < 0.2)
    new = {"append": _log_int(rng, 1, 8192), "step": 1, "few": rng.randint(2, 8), "chunk": _log_int(rng, 9, 8192)}[kind]
    while B > 1 and B * new * kv_heads * D > MAX_NEW:
        B //= 2
    new = max(1, min(new, MAX_NEW // (kv_heads * D)))
    while B > 1 and B * (before + new) * kv_heads * D > MAX_CELLS:
        B //= 2
    before = max(0, min(before, MAX_CELLS // (kv_heads * D) - new))
    more = dict(page=page, rot=rot, interleaved=rng.random() < 0.3, per_head=rng.random() < 0.3, first=rng.choice([0, 0, rng.randint(1, 600)]), mix=mix)
    if kind == "append":
        return _append(None, B, q_heads, kv_heads, D, (max(1, new // 20), new), (before // 20, before), **more)
    window, sinks = _log_int(rng, 16, 8192), _log_int(rng, 1, 256)
    seen = lambda: min(before + new, window + new + sinks)
    while B > 1 and (B * q_heads * new * seen() > MAX_SCORES or B * seen() * kv_heads * D > MAX_SEEN):
        B //= 2
    while q_heads * new * seen() > MAX_SCORES:
        new //= 2
    while seen() * kv_heads * D > MAX_SEEN:
        window //= 2
    return _stream(None, B, q_heads, kv_heads, D, (max(1, new // 20), new), (before // 20, before), max(1, window), sinks, **more)


def _pairs(case, a, b, count):
    """`count` pairs of numbers within the case's ranges a and b; the first pair has the most of both."""
    rng = random.Random(case["mix"] * 1000003 + case["B"])
    got = [(case[a + "_hi"], case[b + "_hi"])]
    for _ in range(count - 1):
        got.append((rng.randint(case[a + "_lo"], case[a + "_hi"]), rng.randint(case[b + "_lo"], case[b + "_hi"])))
    return got


def _lengths(case):
    """[(tokens held before, new tokens)] of the sequences (of branches: of the children, the tokens that their parent holds)."""
    if case["kind"] != "branch":
        return _pairs(case, "before", "new", case["B"])
    parents = [b for b, _ in _pairs(case, "before", "new", case["B"])]
    rng = random.Random(case["mix"] * 7 + 1)
    return [(parents[i // case["children"]], case["new_hi"] if i == 0 else rng.randint(case["new_lo"], case["new_hi"])) for i in range(case["B"] * case["children"])]


def _moves(case):
    """[(tokens held, tokens kept, tokens before them at the new place)] of the sequences."""
    rng = random.Random(case["mix"] * 11 + 5)
    return [(held, min(kept, held, 64 if case["choice"] == "tail" else held), case["to_hi"] if i == 0 else rng.randint(case["to_lo"], case["to_hi"]))
            for i, (held, kept) in enumerate(_pairs(case, "held", "kept", case["B"]))]


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


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)


def _tables(gen, counts, width, extra):
    """Tables [len(counts)][width] of counts pages each, anywhere among all (extra: pages of none), -1 behind them; and how many pages there are."""
    pages = sum(counts) + extra
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    n = _i32(counts).long()
    e = torch.arange(width, device=DEV)
    place = (n.cumsum(0) - n)[:, None] + e
    return torch.where(e < n[:, None], order[place.clamp(max=pages - 1)], -1).contiguous(), pages


def _cache(gen, pages, H, D, P, loud):
    """Pages full of keys and values: codes and scale bytes, the keys' and the values'; blocks differ in scale, keys have a few channels that are larger."""
    got = []
    for gain in (loud, 1.0):
        codes = torch.empty(pages, H, P // 32, 32, D, dtype=torch.uint8, device=DEV)
        scales = torch.empty(pages, H, P // 32, dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 28) // (H * P * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = _normal(gen, n, H, P // 32, 32, D) * gain * torch.exp2(torch.rand(n, H, P // 32, 1, 1, generator=gen, device=DEV) - 0.5)
            byte = _scale_byte(x.abs().amax(dim=(-1, -2)))
            codes[p:p + n] = _e4m3(x * _pow2(127 - byte)[..., None, None])
            scales[p:p + n] = byte.to(torch.uint8)
        got += [codes, scales]
    return got[0], got[1], _values_in_order(got[2]).contiguous(), got[3]


def _rope(most, r):
    """Cosines and sines fp32 [most][r] of the angles p * 10000^(-2 i / r)."""
    angle = torch.arange(most, device=DEV, dtype=torch.float64)[:, None] * torch.exp2(-math.log2(10000.0) * 2.0 / r * torch.arange(r // 2, device=DEV, dtype=torch.float64))
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().contiguous()


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    H, D, P = case["kv_heads"], case["D"], case["page"]
    need = lambda n: (n + P - 1) // P
    loud = 1.0 + 3.0 * (torch.rand(H, 1, 1, D, generator=gen, device=DEV) < 0.02).float()
    s = {"case": dict(case)}
    if case["kind"] == "compact":
        moves = _moves(case)
        held, kept, to = [m[0] for m in moves], [m[1] for m in moves], [m[2] for m in moves]
        width = max(need(n) for n in held)
        to_width = max(need(t + n) for t, n in zip(to, kept))
        both, pages = _tables(gen, [need(n) for n in held] + [need(t + n) for t, n in zip(to, kept)], max(width, to_width), 2)
        s["from_table"], s["to_table"] = both[:case["B"], :width].contiguous(), both[case["B"]:, :to_width].contiguous()
        rows = H if case["choice"] == "heads" else 1
        chosen = []
        for n, k in zip(held, kept):      # ascending
            if case["choice"] == "recent":
                few = min(4, k)
                one = torch.cat([torch.arange(few, device=DEV), torch.arange(n - k + few, n, device=DEV)])[None]
            elif case["choice"] == "tail":
                tail = min(n, 64)
                one = n - tail + torch.randperm(tail, generator=gen, device=DEV)[:k].sort().values[None]
            else:
                one = torch.rand(rows, n, generator=gen, device=DEV).argsort(dim=1)[:, :k].sort(dim=1).values
            chosen.append(one.int())
        s["from_token"] = torch.cat(chosen, dim=1).contiguous()
        cu, start = _starts(kept), [t // 32 * 32 for t in to]
        cu_rows = _starts([t + k - f for t, k, f in zip(to, kept, start)])
        s |= {"cu": _i32(cu), "to": _i32(to), "moves": cu[-1], "start": _i32(start), "cu_rows": _i32(cu_rows), "rows": cu_rows[-1],
              "rope": _rope(max(max(held), max(t + k for t, k in zip(to, kept))), case["rot"]) if case["rot"] else None}
    else:
        lengths = _lengths(case)
        before, new = [b for b, _ in lengths], [n for _, n in lengths]
        cu = _starts(new)
        s |= {"cu": _i32(cu), "T": cu[-1], "max_new": max(new), "max_len": max(b + n for b, n in lengths)}
        if case["kind"] == "branch":
            parents = before[::case["children"]]
            width = max(need(b + n) for b, n in lengths)
            # what all children need beside the pages of their parents, and some more
            own_pages = sum(need(b + n) - b // P for b, n in lengths)
            s["table"], pages = _tables(gen, [need(b) for b in parents], width, max(0, own_pages + case["spare"]))
            named = torch.bincount(s["table"][s["table"] >= 0].long(), minlength=pages)
            s |= {"refs": named.int(), "length": _i32(parents), "parent": _i32([i // case["children"] for i in range(len(new))]), "new": _i32(new),
                  "child_table": torch.full((len(new), width), -1, dtype=torch.int32, device=DEV), "child_length": _i32([0] * len(new)), "missing": _i32([0])}
        else:
            s["table"], pages = _tables(gen, [need(b + n) for b, n in lengths], max(need(b + n) for b, n in lengths), 2)
            Hq, T = case["q_heads"], cu[-1]
            # what the QKV layer leaves: one row a token, queries, keys and values of all heads behind each other
            qkv = _normal(gen, T, (Hq + 2 * H), D)
            qkv[:, Hq:Hq + H] *= loud.view(H, D)
            weights = lambda heads: 0.5 + torch.rand(*((heads, D) if case["per_head"] else (D,)), generator=gen, device=DEV)
            s |= {"qkv": qkv.to(torch.bfloat16), "q_weight": weights(Hq), "k_weight": weights(H), "q_first": weights(Hq), "k_first": weights(H),
                  "rope": _rope(s["max_len"], case["rot"]), "kv_len": _i32([b + n for b, n in lengths])}
            start = [b // 32 * 32 for b in before]
            cu_rows = _starts([b + n - f for (b, n), f in zip(lengths, start)])
            s |= {"start": _i32(start), "cu_rows": _i32(cu_rows), "rows": cu_rows[-1]}
    s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"] = _cache(gen, pages, H, D, P, loud)
    if case["kind"] == "stream":
        s["out"] = torch.empty(s["T"], case["q_heads"], D, dtype=torch.bfloat16, device=DEV)
    elif case["kind"] != "branch":      # rows that are read back
        s["rows_out"] = [torch.empty(s["rows"], H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _branch_outputs(s):
    return {k: s[k] for k in ("child_table", "child_length", "refs", "missing", "k_codes", "k_scales", "v_codes", "v_scales")}


def _run_own(s):
    c = s["case"]
    kind, H = c["kind"], c["kv_heads"]
    if "cache" not in s:      # a program keeps these
        KV = _kv()
        s["cache"] = KV.KVCache.from_buffers(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
        if kind == "compact":
            s["plan"] = KV.KVMoves(s["cu"], s["from_token"], s["to"], s["from_table"], s["to_table"], s["moves"])
            s["rotation"] = KV.Rope(s["rope"], interleaved=c["interleaved"]) if c["rot"] else None
            s["workspace"] = s["cache"].compact_workspace(s["plan"]) if c["staged"] else None
            s["rows_batch"] = KV.KVRows(s["start"], s["cu_rows"], s["to_table"], s["rows"])
        elif kind == "branch":
            s["pool"] = KV.KVPages.from_counts(s["refs"], c["page"])
            s["batch"] = KV.KVBatch(s["cu"], s["child_length"], s["child_table"], s["T"], s["max_new"], s["max_len"])
            s["workspace"] = s["pool"].reserve_workspace(s["batch"])
        else:
            s["batch"] = KV.KVBatch(s["cu"], s["kv_len"], s["table"], s["T"], s["max_new"], s["max_len"])
            s["rotation"] = KV.Rope(s["rope"], interleaved=c["interleaved"])
            s["norm"] = KV.KVNorm(s["q_weight"], s["k_weight"], EPS, q_first=s["q_first"], k_first=s["k_first"], first_tokens=c["first"])
            s["rows_batch"] = KV.KVRows(s["start"], s["cu_rows"], s["table"], s["rows"])
            s["workspace"] = s["cache"].attention_workspace(s["batch"], c["q_heads"]) if kind == "stream" else None
    if kind == "stream":
        return s["cache"].attention(s["qkv"][:, :c["q_heads"]], s["batch"], rope=s["rotation"], window=c["window"], sinks=c["sinks"], norm=s["norm"], out=s["out"],
                                    workspace=s["workspace"])
    if kind == "branch":
        s["pool"].release(s["child_table"])      # the branches of the step before
        s["pool"].fork(s["table"], s["length"], s["parent"], s["child_table"], s["child_length"])
        s["child_length"].add_(s["new"])
        s["pool"].reserve(s["cache"], s["batch"], s["missing"], workspace=s["workspace"])
        return _branch_outputs(s)
    if kind == "append":
        Hq = c["q_heads"]
        s["cache"].append(s["qkv"][:, Hq:Hq + H], s["qkv"][:, Hq + H:], s["batch"], rope=s["rotation"], norm=s["norm"])
    else:
        s["cache"].compact(s["plan"], rope=s["rotation"], workspace=s["workspace"])
    return s["cache"].gather(s["rows_batch"], out=s["rows_out"])


def _turn(x, co, si, interleaved):
    """x [..., D] with the cosines and sines [..., r / 2] of its pairs"""
    r = 2 * co.shape[-1]
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * co - b * si, b * co + a * si], dim=-1).flatten(-2)
    else:
        a, b = x[..., : r // 2], x[..., r // 2:r]
        turned = torch.cat([a * co - b * si, b * co + a * si], dim=-1)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _ready(s, x, weight, first, t):
    """x [token][head][D] at positions t normalised and rotated, in 32 bits"""
    x = x.float()
    if weight.dim() == 1:
        weight, first = weight[None], first[None]
    w = torch.where((t < s["case"]["first"])[:, None, None], first, weight)
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    r = s["case"]["rot"]
    return _turn(x, s["rope"][t, : r // 2][:, None], s["rope"][t, r // 2:][:, None], s["case"]["interleaved"])


def _spread(cu, total):
    """sequence and number within it of every item"""
    n = (cu[1:] - cu[:-1]).long()
    b = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=total)
    return b, torch.arange(total, device=DEV) - cu.long()[b]


def _held(s, page, head, block, at):
    """keys and values fp32 [..., D] of tokens, by index tensors of one shape"""
    slot, j = 2 * (at // 16) + at % 8 // 4, 4 * (at % 16 // 8) + at % 4
    k = s["k_codes"].view(torch.float8_e4m3fn)[page, head, block, at].float() * _pow2(s["k_scales"][page, head, block].int() - 127)[..., None]
    v = s["v_codes"][page, head, block, :, :, slot, :, j].transpose(-1, -2).reshape(k.shape).contiguous()
    return k, v.view(torch.float8_e4m3fn).float() * _pow2(s["v_scales"][page, head, block].int() - 127)[..., None]


def _store(s, table, b, t, first, some, k, v):
    """Quantizes rows fp32 [item][head][D] into positions t of sequences b; `some`: sequences that hold tokens in the block of their first item, at position `first`."""
    D, P = s["case"]["D"], s["case"]["page"]
    H, blocks = k.shape[1], P // 32
    page, block, at = table[b, t // P], t % P // 32, t % 32
    page0, block0 = table.gather(1, (first // P).clamp(max=table.shape[1] - 1)[:, None])[:, 0].clamp(min=0), first % P // 32
    held = torch.zeros(s["k_scales"].shape[0], blocks, dtype=torch.bool, device=DEV)
    held[page0[some], block0[some]] = True
    bad = ~(torch.isfinite(k).all(-1) & torch.isfinite(v).all(-1))
    for x, codes, scales, empty in ((k, s["k_codes"], s["k_scales"], float("nan")), (v, s["v_codes"], s["v_scales"], 0.0)):
        amax = torch.where(bad, torch.zeros((), device=DEV), x.abs().amax(-1))
        top = torch.zeros(scales.shape[0] * blocks, H, device=DEV).index_reduce_(0, page * blocks + block, amax, "amax")
        byte = _scale_byte(top)[page * blocks + block]                                       # [item][head]
        byte = torch.maximum(byte, torch.where(held[page, block][:, None], scales[page, :, block].int(), 0))
        was = scales[page0, :, block0].int()                                                 # of the first blocks, before
        scales[page, :, block] = byte.to(torch.uint8)
        # what the first blocks hold, at the scale that they have now
        now = scales[page0, :, block0].int()
        kept = codes[page0, :, block0]                                                       # [sequence][head]...
        wide = lambda z: z.view(*z.shape, *[1] * (kept.dim() - 2))
        again = _e4m3(kept.view(torch.float8_e4m3fn).float() * wide(_pow2((was - now).clamp(min=-100))))
        codes[page0, :, block0] = torch.where(wide(some[:, None] & (now > was)), again, kept)
        fresh = _e4m3(torch.where(bad[..., None], empty, x * _pow2(127 - byte)[..., None]))
        if codes is s["k_codes"]:
            codes[page, :, block, at] = fresh
        else:
            codes[page, :, block, :, :, 2 * (at // 16) + at % 8 // 4, :, 4 * (at % 16 // 8) + at % 4] = fresh.view(*fresh.shape[:2], D // 32, 2, 16).transpose(-1, -2)


def _read_back(s, table):
    b, i = _spread(s["cu_rows"], s["rows"])
    t, P = i + s["start"].long()[b], s["case"]["page"]
    head = torch.arange(s["case"]["kv_heads"], device=DEV)[None]
    k, v = _held(s, table[b, t // P][:, None], head, (t % P // 32)[:, None], (t % 32)[:, None])
    s["rows_out"][0].copy_(k)
    s["rows_out"][1].copy_(v)
    return s["rows_out"]


def _run_plain(s):
    c = s["case"]
    kind, H, P = c["kind"], c["kv_heads"], c["page"]
    if kind == "stream":
        return _stream_plain(s)
    if kind == "branch":
        return _branch_plain(s)
    if kind == "append":
        Hq, table = c["q_heads"], s["table"].long()
        b, i = _spread(s["cu"], s["T"])
        new = (s["cu"][1:] - s["cu"][:-1]).long()
        first = s["kv_len"].long() - new
        t = first[b] + i
        _store(s, table, b, t, first, (first % 32 > 0) & (new > 0), _ready(s, s["qkv"][:, Hq:Hq + H], s["k_weight"], s["k_first"], t), s["qkv"][:, Hq + H:].float())
        return _read_back(s, table)
    table, to = s["from_table"].long(), s["to"].long()
    b, i = _spread(s["cu"], s["moves"])
    old, t = s["from_token"].long().T, to[b] + i                                # [move][1 or head]
    k, v = _held(s, table[b[:, None], old // P], torch.arange(H, device=DEV)[None], old % P // 32, old % 32)
    if c["rot"]:
        r = c["rot"]
        c0, s0, c1, s1 = s["rope"][old, : r // 2], s["rope"][old, r // 2:], s["rope"][t, : r // 2][:, None], s["rope"][t, r // 2:][:, None]
        size = c0 * c0 + s0 * s0
        k = _turn(k, (c1 * c0 + s1 * s0) / size, (s1 * c0 - c1 * s0) / size, c["interleaved"])
    _store(s, s["to_table"].long(), b, t, to, (to % 32 > 0) & (s["cu"][1:] > s["cu"][:-1]), k, v)
    return _read_back(s, s["to_table"].long())


def _branch_plain(s):
    c = s["case"]
    P, E, S = c["page"], s["child_table"].shape[1], s["child_table"].shape[0]
    refs, table = s["refs"], s["child_table"]
    pages = refs.numel()
    count = lambda named, ok: torch.zeros_like(refs).index_add_(0, named.clamp(0, pages - 1).flatten().long(), ok.flatten().int())
    # the branches of the step before are given back
    refs.sub_(count(table, (table >= 0) & (table < pages)))
    # the children take their parents' pages
    parent, e = s["parent"].long(), torch.arange(E, device=DEV)
    held = s["length"][parent]
    table.copy_(torch.where(e < ((held + P - 1) // P)[:, None], s["table"][parent], -1))
    refs.add_(count(table, (table >= 0) & (table < pages)))
    # those that the new tokens fall in are their own
    length = s["child_length"].copy_(held).add_(s["new"])
    first = (length - s["new"]).clamp(min=0)
    named = (table >= 0) & (table < pages)
    shared = named & (refs[table.clamp(0, pages - 1).long()] > 1)
    lacks = (e >= (first // P)[:, None]) & (e < ((length + P - 1) // P)[:, None]) & (~named | shared)
    rank = lacks.flatten().long().cumsum(0).view(S, E) - 1
    free = (refs <= 0).sum()
    order = torch.argsort((refs > 0).int(), stable=True).int()                  # the free ones first, in order
    served = lacks & (rank < free)
    got = torch.where(served, order[rank.clamp(0, pages - 1)], -1)
    s["missing"].copy_((lacks & ~served).sum().int().view(1))
    # what a shared page holds before the new tokens
    copied = served & named & ((e * P) < first[:, None])
    left, takes = torch.where(lacks, table, -1), copied.any(1)
    at = copied.int().argmax(1)[:, None]
    source = torch.where(takes, table.gather(1, at)[:, 0], 0).long()
    target = torch.where(takes, got.gather(1, at)[:, 0], 0).long()
    inside = torch.where(takes, (first - at[:, 0] * P + 31) // 32, 0)
    child, block = torch.nonzero(torch.arange(P // 32, device=DEV) < inside[:, None], as_tuple=True)
    for x in (s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"]):
        x[target[child], :, block] = x[source[child], :, block]
    refs.sub_(count(left, (left >= 0) & (left < pages)))
    refs.add_(count(got, served))
    table.copy_(torch.where(lacks, got, table))
    return _branch_outputs(s)


def _stream_plain(s):
    c = s["case"]
    B, Hq, H, D, P, n = c["B"], c["q_heads"], c["kv_heads"], c["D"], c["page"], s["max_new"]
    g = Hq // H
    b, i = _spread(s["cu"], s["T"])
    length, new = s["kv_len"].long(), (s["cu"][1:] - s["cu"][:-1]).long()
    first = length - new
    q = torch.zeros(B, n, Hq, D, device=DEV)
    q[b, i] = _ready(s, s["qkv"][:, :Hq], s["q_weight"], s["q_first"], first[b] + i)
    q = q.view(B, n, H, g, D).permute(0, 2, 1, 3, 4).reshape(B * H, n * g, D) * (1.0 / math.sqrt(D))
    # the keys that some row sees: the first ones, and from where the first row's window begins
    sinks, wide = min(c["sinks"], s["max_len"]), min(s["max_len"], c["window"] + n - 1)
    lo = (first + 1 - c["window"]).clamp(min=0)
    key = torch.cat([torch.arange(sinks, device=DEV).expand(B, sinks), lo[:, None] + torch.arange(wide, device=DEV)], dim=1)
    real = key < length[:, None]
    real[:, :sinks] &= key[:, :sinks] < lo[:, None]
    L = sinks + wide
    at = key.clamp(max=s["table"].shape[1] * P - 1)
    page = s["table"].long().gather(1, at // P).clamp(min=0)
    k, v = _held(s, page[:, None], torch.arange(H, device=DEV)[None, :, None], (at % P // 32)[:, None], (at % 32)[:, None])
    v.masked_fill_(~real[:, None, :, None], 0.0)
    x = torch.matmul(q, k.reshape(B * H, L, D).transpose(1, 2).contiguous()).view(B, H, n, g, L)
    del k
    p = first[:, None, None] + torch.arange(n, device=DEV)[:, None]
    seen = real[:, None] & (key[:, None] <= p) & ((key[:, None] > p - c["window"]) | (key[:, None] < c["sinks"]))
    x.masked_fill_(~seen.view(B, 1, n, 1, L), float("-inf"))
    x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    x.div_(x.sum(-1, keepdim=True).clamp(min=1e-30))
    o = torch.matmul(x.view(B * H, n * g, L), v.view(B * H, L, D))
    s["out"].copy_(o.view(B, H, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)[b, i])
    return s["out"]


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    H, D, P = case["kv_heads"], case["D"], case["page"]
    nbytes, flops = 0, 0
    if case["kind"] == "compact":
        for held, kept, to in _moves(case):
            rows = to + kept - to // 32 * 32
            nbytes += 4 * kept * H * D + 4 * kept * (H if case["choice"] == "heads" else 1) + 8 * kept * case["rot"] + 2 * rows * H * D + 4 * rows * H * D
            flops += (8 if case["rot"] else 2) * kept * H * D
        return {"bytes": nbytes, "flops": flops}
    if case["kind"] == "branch":
        lengths = _lengths(case)
        width = max((b + n + P - 1) // P for b, n in lengths)
        for before, _ in lengths:
            nbytes += 4 * H * D * ((before % P + 31) // 32 * 32) + 12 * width
        pages = sum((b + P - 1) // P for b, _ in lengths[::case["children"]]) + sum((b + n + P - 1) // P - b // P for b, n in lengths) + case["spare"]
        return {"bytes": nbytes + 8 * pages, "flops": 0}
    for before, new in _lengths(case):
        L = before + new
        if case["kind"] == "stream":
            Hq, w = case["q_heads"], case["window"]
            least = max(0, before + 1 - w)
            cells = L - least + min(case["sinks"], least)
            pairs = sum(min(p + 1, w + min(case["sinks"], max(0, p + 1 - w))) for p in range(before, L))
            nbytes += 2 * cells * H * D + (cells + 31) // 32 * H * 2 + 4 * new * Hq * D + 4 * new * case["rot"]
            flops += 4 * D * Hq * pairs
        else:
            rows = L - before // 32 * 32
            nbytes += 4 * new * H * D + 2 * new * H * D + 4 * new * case["rot"] + 2 * rows * H * D + 4 * rows * H * D
            flops += 7 * new * H * D
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


def _held64(s, row, tokens):
    """keys and values [heads][token][D] of tokens [1 or heads][token] of a table's row, and their scales' exponents"""
    c = s["case"]
    D, P, Hkv = c["D"], c["page"], c["kv_heads"]
    page, block, at = row.long()[tokens // P], tokens % P // 32, tokens % 32
    head = torch.arange(Hkv, device=DEV)[:, None]
    unit = (page * Hkv + head) * (P // 32) + block                          # [head][token]
    d = torch.arange(D, device=DEV)
    at = at.expand(unit.shape)[..., None]
    k = s["k_codes"].view(-1)[unit[..., None] * (32 * D) + (at * D + d)]
    slot, j = 2 * (at // 16) + at % 8 // 4, 4 * (at % 16 // 8) + at % 4
    v = s["v_codes"].view(-1)[unit[..., None] * (32 * D) + ((((d // 32) * 16 + d % 16) * 4 + slot) * 2 + d % 32 // 16) * 8 + j]
    ek, ev = s["k_scales"].view(-1)[unit].long() - 127, s["v_scales"].view(-1)[unit].long() - 127
    return _decode64(k), _decode64(v), ek, ev


def _turn64(x, position, s, back=False):
    """x [..., token, D] turned by the angles of its tokens' positions, or back, in 64 bits"""
    r, y = s["rope"].shape[1], x.clone()
    for i in range(r // 2):
        one, two = (2 * i, 2 * i + 1) if s["case"]["interleaved"] else (i, i + r // 2)
        co, si = s["rope"][position, i].double(), s["rope"][position, r // 2 + i].double()
        if back:
            size = co * co + si * si
            co, si = co / size, -si / size
        y[..., one] = x[..., one] * co - x[..., two] * si
        y[..., two] = x[..., two] * co + x[..., one] * si
    return y


def _ready64(s, x, weight, first, place):
    """x [token][head][D] normalised and rotated, as [head][token][D]"""
    y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    for i in range(y.shape[1]):
        w, f = (weight[i], first[i]) if weight.dim() == 2 else (weight, first)
        y[:, i] *= torch.where((place < s["case"]["first"])[:, None], f.double(), w.double())
    return _turn64(y.transpose(0, 1), place, s)


def _blocks64(fresh, held, old, e_old):
    """What a run of blocks holds [heads][held + new][D]: `held` tokens `old` with exponent `e_old` in the first block, `fresh` behind them."""
    H, new, D = fresh.shape
    span = (held + new + 31) // 32 * 32
    padded = torch.zeros(H, span, D, dtype=torch.float64, device=DEV)
    padded[:, held:held + new] = fresh
    amax = padded.view(H, -1, 32 * D).abs().amax(-1)
    e = torch.ceil(torch.log2((amax / 448).clamp(min=2.0 ** -126)))
    if held:
        e[:, 0] = torch.maximum(e[:, 0], e_old[:, 0].double())
    e = e.repeat_interleave(32, dim=1)[..., None]
    got = _round64(padded * torch.exp2(-e))
    if held:
        got[:, :held] = _round64(old * torch.exp2(e_old.double()[..., None] - e[:, :held]))
    return (got * torch.exp2(e))[:, :held + new].transpose(0, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "branch":
        return _branch_exact(s)
    H, D = case["kv_heads"], case["D"]
    out, at, rows = [], 0, [[], []]
    if case["kind"] == "compact":
        for b, (_, kept, to) in enumerate(_moves(case)):
            tokens = s["from_token"][:, at:at + kept].long()
            at += kept
            k, v, ek, ev = _held64(s, s["from_table"][b], tokens)
            k, v = k * torch.exp2(ek.double())[..., None], v * torch.exp2(ev.double())[..., None]
            if case["rot"]:
                k = _turn64(_turn64(k, tokens.expand(H, kept), s, back=True), torch.arange(to, to + kept, device=DEV), s)
            start = to // 32 * 32
            old = _held64(s, s["to_table"][b], torch.arange(start, to, device=DEV)[None]) if to > start else (None,) * 4
            rows[0].append(_blocks64(k, to - start, old[0], old[2]))
            rows[1].append(_blocks64(v, to - start, old[1], old[3]))
        return [torch.cat(r) for r in rows]
    Hq = case["q_heads"]
    for b, (before, new) in enumerate(_lengths(case)):
        L = before + new
        x = s["qkv"][at:at + new].double()
        at += new
        place = torch.arange(before, L, device=DEV)
        if case["kind"] == "append":
            start = before // 32 * 32
            old = _held64(s, s["table"][b], torch.arange(start, before, device=DEV)[None]) if before > start else (None,) * 4
            rows[0].append(_blocks64(_ready64(s, x[:, Hq:Hq + H], s["k_weight"], s["k_first"], place), before - start, old[0], old[2]))
            rows[1].append(_blocks64(x[:, Hq + H:].transpose(0, 1), before - start, old[1], old[3]))
            continue
        least = max(0, before + 1 - case["window"])
        tokens = torch.cat([torch.arange(min(case["sinks"], least), device=DEV), torch.arange(least, L, device=DEV)])
        k, v, ek, ev = _held64(s, s["table"][b], tokens[None])
        k, v = k * torch.exp2(ek.double())[..., None], v * torch.exp2(ev.double())[..., None]
        q = _ready64(s, x[:, :Hq], s["q_weight"], s["q_first"], place)
        o = torch.zeros(new, Hq, D, dtype=torch.float64, device=DEV)
        step = max(1, (1 << 28) // tokens.numel())
        for h in range(Hq):
            for i in range(0, new, step):
                p = place[i:i + step, None]
                score = q[h, i:i + step] @ k[h // (Hq // H)].T / math.sqrt(D)
                hidden = (tokens > p) | ((tokens <= p - case["window"]) & (tokens >= case["sinks"]))
                o[i:i + step, h] = torch.softmax(score.masked_fill_(hidden, float("-inf")), dim=-1) @ v[h // (Hq // H)]
        out.append(o)
    return [torch.cat(r) for r in rows] if case["kind"] == "append" else torch.cat(out)


def _branch_exact(s):
    """One page after another, on the host; codes and bytes are whole numbers."""
    c = s["case"]
    P = c["page"]
    refs, parents, length = s["refs"].tolist(), s["table"].tolist(), s["length"].tolist()
    new, parent = s["new"].tolist(), s["parent"].tolist()
    children = []
    for p in parent:
        row = [g if e * P < length[p] else -1 for e, g in enumerate(parents[p])]
        for g in row:
            if g >= 0:
                refs[g] += 1
        children.append(row)
    free = [g for g, n in enumerate(refs) if n <= 0]
    was, missing = list(refs), 0
    for row, p, n in zip(children, parent, new):
        before = length[p]
        for e in range(before // P, (before + n + P - 1) // P):
            g = row[e]
            if g >= 0 and was[g] <= 1:
                continue
            if g >= 0:
                refs[g] -= 1
            row[e] = free.pop(0) if free else -1
            missing += row[e] < 0
            if row[e] >= 0:
                refs[row[e]] = 1
                if g >= 0 and e * P < before:
                    for x in (s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"]):
                        x[row[e], :, :(before - e * P + 31) // 32] = x[g, :, :(before - e * P + 31) // 32]
    return {"child_table": _i32(children), "child_length": _i32([length[p] + n for p, n in zip(parent, new)]), "refs": _i32(refs), "missing": _i32([missing]),
            "k_codes": s["k_codes"], "k_scales": s["k_scales"], "v_codes": s["v_codes"], "v_scales": s["v_scales"]}
