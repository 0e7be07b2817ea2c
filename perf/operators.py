"""The live cache beside the coder, as timed cases: tokens written into pages, read back, and attended to by one new token a sequence.

A case is a dict of plain values; "op" picks the operator:

  write    keys and values of new tokens into their slots of a paged cache, quantised on the way
  read     keys and values of slots back as features (what the coder takes when tokens leave the window)
  attend   one new token of every sequence over its pages

Common to all: "format" (how the cache holds values: bf16, fp8 = E4M3 with an fp32 scale per token and head, int4 = 4-bit codes with an fp16
shift and scale per 32 features), "dtype" of the features or queries, "heads" and "d" of the cache, "page" tokens to a page, and "order":
"heads" for pages [heads][page][d], "tokens" for [page][heads][d].
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
GROUP = 32                              # features that share a shift and a scale in the 4-bit format
FORMATS = ("bf16", "fp8", "int4")
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # serving, every generated token: one token of each of 64 caches joins its last page; latency
        {"name": "write_step_fp8", "op": "write", "format": "fp8", "dtype": "bf16", "heads": 8, "d": 128, "page": 64, "order": "heads",
         "tokens": 64, "runs": 64, "padding": 0},
        # a decoded (or prefilled) context of 32768 tokens goes into pages
        {"name": "write_context_fp8", "op": "write", "format": "fp8", "dtype": "bf16", "heads": 8, "d": 128, "page": 64, "order": "heads",
         "tokens": 32768, "runs": 1, "padding": 0},
        # ragged prompts in fp32 into small token-major pages of 4 bits, the end of the batch padded; then read back as the values it stands for
        {"name": "write_prompts_int4", "op": "write", "format": "int4", "dtype": "f32", "heads": 4, "d": 64, "page": 16, "order": "tokens",
         "tokens": 9001, "runs": 13, "padding": 55},
        # every 16 generated tokens of 256 caches: what left the window goes to the coder
        {"name": "read_window_fp8", "op": "read", "format": "fp8", "dtype": "bf16", "heads": 8, "d": 128, "page": 64, "order": "heads",
         "tokens": 4096, "runs": 256, "padding": 0},
        # a whole context of 32768 tokens leaves a 4-bit cache for the coder
        {"name": "read_context_int4", "op": "read", "format": "int4", "dtype": "bf16", "heads": 8, "d": 128, "page": 128, "order": "tokens",
         "tokens": 32768, "runs": 1, "padding": 0},
        # few wide heads in fp32, pages whose size is no power of two, an odd number of tokens
        {"name": "read_odd_bf16", "op": "read", "format": "bf16", "dtype": "f32", "heads": 2, "d": 256, "page": 20, "order": "heads",
         "tokens": 777, "runs": 5, "padding": 33},
        # one user, a short context: latency
        {"name": "attend_short_bf16", "op": "attend", "format": "bf16", "dtype": "bf16", "heads": 8, "queries": 32, "d": 128, "page": 64,
         "order": "heads", "seqs": 1, "shortest": 700, "longest": 700, "pick": 0, "sinks": 0, "window": 0},
        # one user, the long context of 131072 tokens, in 8 bits
        {"name": "attend_long_fp8", "op": "attend", "format": "fp8", "dtype": "bf16", "heads": 8, "queries": 32, "d": 128, "page": 64,
         "order": "heads", "seqs": 1, "shortest": 131072, "longest": 131072, "pick": 0, "sinks": 0, "window": 0},
        # 64 of the ragged batch's caches of 512 to 16384 tokens, 40 query heads
        {"name": "attend_ragged_bf16", "op": "attend", "format": "bf16", "dtype": "bf16", "heads": 8, "queries": 40, "d": 128, "page": 64,
         "order": "heads", "seqs": 64, "shortest": 512, "longest": 16384, "pick": 1, "sinks": 0, "window": 0},
        # 16 contexts of 32768 tokens or a little less in 4 bits
        {"name": "attend_batch_int4", "op": "attend", "format": "int4", "dtype": "bf16", "heads": 8, "queries": 32, "d": 128, "page": 128,
         "order": "tokens", "seqs": 16, "shortest": 30000, "longest": 32768, "pick": 2, "sinks": 0, "window": 0},
        # as many query as KV heads, fp32 queries, small token-major pages, lengths from none on
        {"name": "attend_heads_fp8", "op": "attend", "format": "fp8", "dtype": "f32", "heads": 12, "queries": 12, "d": 64, "page": 16,
         "order": "tokens", "seqs": 24, "shortest": 0, "longest": 4001, "pick": 3, "sinks": 0, "window": 0},
        # streaming: 256 caches, each attends to its 4 sinks and the 128 newest tokens
        {"name": "attend_window_bf16", "op": "attend", "format": "bf16", "dtype": "bf16", "heads": 8, "queries": 32, "d": 128, "page": 16,
         "order": "heads", "seqs": 256, "shortest": 1, "longest": 2048, "pick": 4, "sinks": 4, "window": 128},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    case = {"op": rng.choice(["write", "read", "attend", "attend"]), "format": rng.choice(FORMATS), "dtype": "f32" if rng.random() < 0.25 else "bf16",
            "heads": rng.choice([1, 2, 3, 4, 8, 8, 12, 16]), "d": rng.choice([64, 128, 128, 128, 256]),
            "page": rng.choice([1, 16, 20, 32, 64, 64, 96, 128, 256]), "order": rng.choice(["heads", "tokens"])}
    width = case["heads"] * case["d"]
    if case["op"] != "attend":
        tokens = _log(rng, 1, min(60_000, 33_000_000 // width))
        return {**case, "tokens": tokens, "runs": min(tokens, _log(rng, 1, 256)), "padding": rng.choice([0, 0, 1, tokens // 7])}
    longest = _log(rng, 1, min(131_072, 134_000_000 // width))
    seqs = max(1, min(_log(rng, 1, 256), 134_000_000 // (width * longest)))
    case |= {"queries": case["heads"] * rng.choice([1, 1, 2, 3, 4, 4, 5, 7, 8, 16, 24]), "seqs": seqs, "shortest": rng.choice([0, 1, longest // 32, longest // 2, longest]),
             "longest": longest, "pick": rng.randint(0, 10**6), "sinks": 0, "window": 0}
    if rng.random() < 0.25:
        case |= {"sinks": rng.choice([0, 4, 33]), "window": _log(rng, 1, 2 * longest)}
    return case


# ---- shapes ---------------------------------------------------------------------------------------------------------------

def _lengths(c):
    rng = random.Random(c["pick"])
    lo, hi = c["shortest"], c["longest"]
    if lo == hi:
        return [hi] * c["seqs"]
    at = [int(round(math.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1))))) - 1 for _ in range(c["seqs"])]
    return [min(hi, max(lo, n)) for n in at]


def _seen(c, length):
    """Tokens of a sequence that its new token attends to."""
    return length if not c["window"] else min(length, c["window"] + min(c["sinks"], max(0, length - c["window"])))


def _row_bytes(c):
    return {"bf16": 2 * c["d"], "fp8": c["d"], "int4": c["d"] // 2}[c["format"]]


def _scale_bytes(c):
    return {"bf16": 0, "fp8": 4, "int4": 4 * c["d"] // GROUP}[c["format"]]


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "attend":
        lengths = _lengths(c)
        seen = sum(_seen(c, n) for n in lengths)
        kept = 2 * seen * c["heads"] * (_row_bytes(c) + _scale_bytes(c))
        table = 4 * sum(-(-_seen(c, n) // c["page"]) + 1 for n in lengths)
        return {"bytes": kept + table + c["seqs"] * c["queries"] * (2 * c["d"] * e + 4), "flops": 4 * seen * c["queries"] * c["d"]}
    n = c["tokens"] - c["padding"]
    kept, features = 2 * n * c["heads"] * (_row_bytes(c) + _scale_bytes(c)), 2 * n * c["heads"] * c["d"]
    if c["op"] == "read":
        return {"bytes": kept + e * 2 * c["tokens"] * c["heads"] * c["d"] + 8 * c["tokens"], "flops": features}
    moved = kept + e * features + 8 * c["tokens"]
    if c["format"] == "int4":                       # with the values read back
        moved += kept + 4 * 2 * c["tokens"] * c["heads"] * c["d"] + 8 * c["tokens"]
    return {"bytes": moved, "flops": 4 * features}


# ---- the formats, in elementary operations --------------------------------------------------------------------------------

def _half_directed(x, up):
    """fp32 to fp16 towards +inf or -inf, at most +-65504."""
    x = x.clamp(-65504.0, 65504.0)
    h = x.to(torch.float16)
    bits = h.view(torch.int16).to(torch.int32)
    key = torch.where(bits >= 0, bits, -(bits & 0x7FFF))
    back = h.to(torch.float32)
    key = key + ((back < x).to(torch.int32) if up else -(back > x).to(torch.int32))
    return torch.where(key >= 0, key, -key - 32768).to(torch.int16).view(torch.float16)


def _quantise(x, fmt):
    """Rows [..., d] in fp32: (what the cache's rows hold, its scales)."""
    if fmt == "bf16":
        return x.to(torch.bfloat16), None
    if fmt == "fp8":
        scale = x.abs().amax(-1, keepdim=True) / 448.0
        scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
        inverse = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
        return (x * inverse).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale[..., 0]
    g = x.unflatten(-1, (-1, GROUP))
    shift = _half_directed(g.amin(-1), False)
    scale = _half_directed((g.amax(-1) - shift.to(torch.float32)) / 15.0, True)
    s = scale.to(torch.float32)
    inverse = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    codes = ((g - shift.to(torch.float32)[..., None]) * inverse[..., None]).round().clamp(0.0, 15.0).to(torch.uint8)
    pairs = codes.unflatten(-1, (GROUP // 2, 2))                                    # [..., group, pair, 2]
    packed = (pairs[..., 0] | (pairs[..., 1] << 4)).transpose(-1, -2).flatten(-2)    # byte pair * groups + group
    return packed, torch.stack([shift, scale], -1)


def _values(rows, scales, fmt):
    """The opposite: fp32 values of rows as the cache holds them."""
    if fmt == "bf16":
        return rows.to(torch.float32)
    if fmt == "fp8":
        return rows.view(torch.float8_e4m3fn).to(torch.float32) * scales[..., None]
    packed = rows.unflatten(-1, (GROUP // 2, -1)).transpose(-1, -2)
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).to(torch.float32)
    header = scales.to(torch.float32)
    return (codes * header[..., 1:2] + header[..., 0:1]).flatten(-2)


# ---- inputs ---------------------------------------------------------------------------------------------------------------

def _features(gen, shape):
    """Keys or values: normal, with a mean of each channel and a few channels of ten times the size."""
    x = torch.randn(shape, generator=gen, device=DEV)
    size = torch.ones(shape[-2:], device=DEV)
    size[:, ::29] = 4.0
    return x * size + 0.5 * torch.randn(shape[-2:], generator=gen, device=DEV)


def _pool(c, n_pages, gen):
    """The rows and scales of all pages, filled: [pages][heads][page][...] or [pages][page][heads][...], scales always heads first."""
    fmt, h, d, p = c["format"], c["heads"], c["d"], c["page"]
    dtype, width = (torch.bfloat16, d) if fmt == "bf16" else (torch.uint8, _row_bytes(c))
    rows = torch.empty((n_pages, h, p, width) if c["order"] == "heads" else (n_pages, p, h, width), dtype=dtype, device=DEV)
    scales = {"bf16": None, "fp8": torch.empty((n_pages, h, p), device=DEV) if fmt == "fp8" else None,
              "int4": torch.empty((n_pages, h, p, d // GROUP, 2), dtype=torch.float16, device=DEV) if fmt == "int4" else None}[fmt]
    step = max(1, (1 << 25) // (h * p * d))
    for at in range(0, n_pages, step):
        n = min(step, n_pages - at)
        r, s = _quantise(_features(gen, (n, p, h, d)).to(torch.bfloat16).to(torch.float32), fmt)
        rows[at:at + n] = r.transpose(1, 2) if c["order"] == "heads" else r
        if s is not None:
            scales[at:at + n] = s.transpose(1, 2)
    return rows, scales


def _slots(c, gen):
    """A slot for every token: runs of tokens side by side, each from somewhere in a page of its own on; the last ones of the batch nowhere."""
    p, runs = c["page"], c["runs"]
    each = -(-c["tokens"] // runs)
    pages_each = -(-each // p) + 1
    n_pages = runs * pages_each
    order = torch.randperm(n_pages, generator=gen, device=DEV).view(runs, pages_each)
    first = torch.randint(0, p, (runs, 1), generator=gen, device=DEV)
    place = first + torch.arange(each, device=DEV)
    slots = (torch.gather(order, 1, place // p) * p + place % p).flatten()[:c["tokens"]].clone()
    if c["padding"]:
        slots[-c["padding"]:] = -1
    return slots, n_pages


def prepare(c, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(c)
    dtype = DTYPES[c["dtype"]]
    if c["op"] == "attend":
        lengths, p = _lengths(c), c["page"]
        pages = [-(-n // p) for n in lengths]
        n_pages, widest = max(1, sum(pages)), max(1, max(pages))
        order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
        table = torch.full((c["seqs"], widest), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = order[at:at + n]
            at += n
        q = torch.randn((c["seqs"], c["queries"], c["d"]), generator=gen, device=DEV).to(dtype)
        s |= {"table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device=DEV), "longest_now": max(lengths), "q": q, "out": torch.empty_like(q),
              "lse": torch.empty((c["seqs"], c["queries"]), device=DEV), "factor": c["d"] ** -0.5}
    else:
        s["slots"], n_pages = _slots(c, gen)
        shape = (c["tokens"], c["heads"], c["d"])
        if c["op"] == "write":
            s["k"], s["v"] = _features(gen, shape).to(dtype), _features(gen, shape).to(dtype)
        if c["op"] == "read" or c["format"] == "int4":
            out = dtype if c["op"] == "read" else torch.float32
            s["k_out"], s["v_out"] = torch.empty(shape, dtype=out, device=DEV), torch.empty(shape, dtype=out, device=DEV)
    s["pages"] = n_pages
    s["k_rows"], s["k_scales"] = _pool(c, n_pages, gen)
    s["v_rows"], s["v_scales"] = _pool(c, n_pages, gen)
    if own:                                         # the descriptor of the cache and the workspace, which a serving program keeps
        import paper_2511_01815_amd as kv
        rows = s["k_rows"]
        page, head, token = [rows.stride(i) * rows.element_size() for i in ((0, 1, 2) if c["order"] == "heads" else (0, 2, 1))]
        s["kv"] = kv
        s["cache"] = kv.cache({"bf16": kv.KVTC_CACHE_BF16, "fp8": kv.KVTC_CACHE_FP8, "int4": kv.KVTC_CACHE_INT4}[c["format"]], n_pages, c["page"], c["heads"], c["d"],
                              s["k_rows"], s["v_rows"], page, head, token, s["k_scales"], s["v_scales"])
        s["type"] = kv.KVTC_BF16 if c["dtype"] == "bf16" else kv.KVTC_F32
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if c["op"] == "attend":
            s["work"] = torch.zeros(kv.kvtc_attend_work_bytes(s["cache"], c["seqs"], c["queries"], max(1, s["longest_now"])), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------------

def _gather(s, rows, scales, page, place):
    """fp32 values [..., heads, d] of the tokens at `place` of `page`."""
    r = rows.transpose(1, 2) if s["order"] == "heads" else rows
    return _values(r[page, place], None if scales is None else scales.transpose(1, 2)[page, place], s["format"])


def _write_plain(s):
    slots, p = s["slots"], s["page"]
    fine = slots >= 0
    page, place = slots[fine] // p, slots[fine] % p
    for side in ("k", "v"):
        rows, scales = _quantise(s[side][fine].to(torch.float32), s["format"])
        pool = s[side + "_rows"]
        (pool.transpose(1, 2) if s["order"] == "heads" else pool)[page, place] = rows
        if scales is not None:
            s[side + "_scales"].transpose(1, 2)[page, place] = scales


def _read_plain(s, dtype):
    slots, p = s["slots"], s["page"]
    at = slots.clamp(min=0)
    fine = (slots >= 0)[:, None, None]
    k, v = [_gather(s, s[side + "_rows"], s[side + "_scales"], at // p, at % p) for side in ("k", "v")]
    zero = torch.zeros((), device=DEV)
    return torch.where(fine, k, zero).to(dtype), torch.where(fine, v, zero).to(dtype)


def _attend_plain(s):
    n, p, h = s["longest_now"], s["page"], s["heads"]
    b, hq, d = s["q"].shape
    t = torch.arange(max(1, n), device=DEV)
    length = s["lengths"][:, None]
    seen = t < length
    if s["window"]:
        seen &= (t < s["sinks"]) | (t >= length - s["window"])
    page = torch.gather(s["table"], 1, (t // p)[None].expand(b, -1)).clamp(min=0).long()
    place = (t % p)[None].expand(b, -1)
    mask = seen[:, None, None, :]
    k = _gather(s, s["k_rows"], s["k_scales"], page, place)
    q = s["q"].to(torch.float32).view(b, h, hq // h, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1)) * s["factor"]
    del k
    score = torch.where(mask, score, torch.full((), -math.inf, device=DEV))
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = torch.exp(score - top)
    total = e.sum(-1, keepdim=True)
    v = torch.where(seen[:, :, None, None], _gather(s, s["v_rows"], s["v_scales"], page, place), torch.zeros((), device=DEV))
    out = torch.matmul(e, v.permute(0, 2, 1, 3))
    out = torch.where(total > 0, out / total, torch.zeros((), device=DEV))
    return out.view(b, hq, d).to(s["q"].dtype), (top + torch.log(total)).view(b, hq)


def run(s):
    op, fmt = s["op"], s["format"]
    if op == "attend":
        if not own:
            return _attend_plain(s)
        s["kv"].kvtc_attend(s["cache"], s["q"], s["type"], s["seqs"], s["queries"], s["queries"] * s["d"], s["d"], s["table"], s["table"].shape[1], s["lengths"],
                            max(1, s["longest_now"]), s["factor"], s["sinks"], s["window"], s["out"], s["lse"], s["work"], s["work"].numel(), s["status"])
        return s["out"], s["lse"]
    wide = s["heads"] * s["d"]
    if op == "read":
        if not own:
            return _read_plain(s, s["k_out"].dtype)
        s["kv"].kvtc_cache_read(s["cache"], s["slots"], s["tokens"], s["k_out"], s["v_out"], s["type"], wide, s["d"], s["status"])
        return s["k_out"], s["v_out"]
    if own:
        s["kv"].kvtc_cache_write(s["cache"], s["k"], s["v"], s["type"], s["tokens"], wide, s["d"], s["slots"], s["status"])
    else:
        _write_plain(s)
    if fmt == "bf16":
        return s["k_rows"], s["v_rows"]
    if fmt == "fp8":
        return s["k_rows"].view(torch.float8_e4m3fn), s["v_rows"].view(torch.float8_e4m3fn), s["k_scales"], s["v_scales"]
    if not own:                                     # 4 bits are no type: the written tokens are read back
        return _read_plain(s, torch.float32)
    s["kv"].kvtc_cache_read(s["cache"], s["slots"], s["tokens"], s["k_out"], s["v_out"], s["kv"].KVTC_F32, wide, s["d"], s["status"])
    return s["k_out"], s["v_out"]


# ---- the definitions, in 64 bits ------------------------------------------------------------------------------------------

def _grid64(x, bits, lowest, how):
    """x onto floating point of `bits` fraction bits and least exponent `lowest`."""
    exponent = (torch.frexp(x).exponent - 1).clamp(min=lowest)
    step = torch.ldexp(torch.ones_like(x), exponent - bits)
    return how(x / step) * step


def _code64(x, fmt):
    """([codes], [scales]) of float64 rows by definition; 4-bit rows: the values they stand for instead."""
    if fmt == "fp8":
        scale = x.abs().amax(-1, keepdim=True) / 448.0
        y = torch.where(scale > 0, x / scale, torch.zeros_like(x))
        return _grid64(y, 3, -6, torch.round).clamp(-448.0, 448.0), scale[..., 0]
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    shift = _grid64(low, 10, -14, torch.floor).clamp(-65504.0, 65504.0)
    scale = _grid64((high - shift) / 15.0, 10, -14, torch.ceil).clamp(max=65504.0)
    code = torch.where(scale > 0, torch.round((g - shift) / scale), torch.zeros_like(g)).clamp(0, 15)
    return (shift + code * scale).reshape(x.shape), None


def _token64(s, side, page, place):
    """Float64 values [n, heads, d] of n tokens, from the bytes of the pool."""
    rows, scales, fmt = s[side + "_rows"], s[side + "_scales"], s["format"]
    r = rows[page, :, place] if s["order"] == "heads" else rows[page, place]
    if fmt == "bf16":
        return r.double()
    if fmt == "fp8":
        b = r.int()
        e, m = (b >> 3) & 15, (b & 7).double()
        size = torch.where(e == 0, m * 2.0 ** -9, torch.ldexp(1 + m / 8, e - 7))
        return torch.where(b >= 128, -size, size) * scales[page, :, place].double()[..., None]
    f = torch.arange(s["d"], device=DEV)
    groups = s["d"] // GROUP
    byte = (f % GROUP) // 2 * groups + f // GROUP
    code = (r[..., byte].int() >> (4 * (f % 2))) & 15
    header = scales[page, :, place][:, :, f // GROUP].double()
    return header[..., 0] + header[..., 1] * code.double()


def exact(c, seed):
    s = prepare(c, seed)
    p, fmt = s["page"], s["format"]
    if s["op"] == "attend":
        per = s["queries"] // s["heads"]
        out = torch.zeros((s["seqs"], s["queries"], s["d"]), dtype=torch.float64, device=DEV)
        lse = torch.full((s["seqs"], s["queries"]), -math.inf, dtype=torch.float64, device=DEV)
        for b, length in enumerate(_lengths(c)):
            t = torch.arange(length, device=DEV)
            if s["window"]:
                t = t[(t < s["sinks"]) | (t >= length - s["window"])]
            if not t.numel():
                continue
            page, place = s["table"][b].long()[t // p], t % p
            k, v = _token64(s, "k", page, place), _token64(s, "v", page, place)
            for h in range(s["heads"]):
                at = slice(h * per, h * per + per)
                score = s["q"][b, at].double() @ k[:, h].T * float(s["factor"])
                lse[b, at] = torch.logsumexp(score, -1)
                out[b, at] = torch.softmax(score, -1) @ v[:, h]
        return out, lse
    slots = s["slots"]
    fine = slots >= 0
    page, place = slots[fine] // p, slots[fine] % p
    if s["op"] == "read" or fmt == "int4":
        got = []
        for side in ("k", "v"):
            out = torch.zeros((s["tokens"], s["heads"], s["d"]), dtype=torch.float64, device=DEV)
            out[fine] = _token64(s, side, page, place) if s["op"] == "read" else _code64(s[side][fine].double(), "int4")[0]
            got.append(out)
        return tuple(got)
    rows, scales = [], []
    for side in ("k", "v"):
        pool = s[side + "_rows"]
        pool = (pool if fmt == "bf16" else pool.view(torch.float8_e4m3fn)).double()
        x = s[side][fine].double()
        if fmt == "fp8":
            x, scale = _code64(x, fmt)
            full = s[side + "_scales"].double()
            full[page, :, place] = scale
            scales.append(full)
        if s["order"] == "heads":
            pool[page, :, place] = x
        else:
            pool[page, place] = x
        rows.append(pool)
    return tuple(rows + scales)
