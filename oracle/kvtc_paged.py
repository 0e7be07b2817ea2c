"""The live cache in pages and the attention over it on the CPU -- TEST INFRASTRUCTURE, NOT A PRODUCT PATH.

What stands beside the coder of "KV Cache Transform Coding for Compact Storage in LLM Inference" in a serving program: keys
and values of new tokens written into pages in 16, 8 or 4 bits, read back, and attended to by one new token of every
sequence.  Everything is the plainest definition available: a row's codes by a search in the table of all E4M3 values or by
the coder's own group quantiser, values and attention in float64, one sequence and head at a time.  Shares no code with the GPU
library and imports nothing from it.

Readings (the paper fixes none of these):
  * 8 bits: E4M3 codes of x * (1 / scale), scale = (largest finite magnitude of the row) * (1 / 448), each a single float32
    operation; scales below 2^-126 count as 0 (all codes 0); NaN keeps its code, infinities give +-448;
  * 4 bits: the coder's min-max quantiser (kvtc_oracle.quantise_group at 4 bits) over every 32 features, but for the range,
    which is multiplied by float32 1 / 15 instead of divided by 15; value = shift + code * scale;
    byte pair * (d / 32) + group of a row holds features 2 * pair (low four bits) and 2 * pair + 1 of the group;
  * a softmax over no tokens, or over scores of minus infinity alone, gives zeros and a log-sum of minus infinity.

Pins (tests/test_oracle_paged.py): codes against the sinks' FP8 oracle and the coder's quantiser, packing against hand-packed
rows, attention against closed forms (equal keys, one token, joined halves).
"""
from __future__ import annotations

import numpy as np

import kvtc_oracle as ko
import kvtc_window as kw

GROUP = 32
_POS = kw.e4m3_table()[:0x7F]                                   # 0 .. 448, ascending


def bf16_bits(x32: np.ndarray) -> np.ndarray:
    """bf16 bit patterns of float32 values, to nearest even; NaN stays NaN."""
    u = np.ascontiguousarray(x32, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x32), np.uint16(0x7FC0), r)


def bf16_value(bits: np.ndarray) -> np.ndarray:
    return (bits.astype(np.uint32) << 16).view(np.float32)


def e4m3_codes(x: np.ndarray) -> np.ndarray:
    """kvtc_window.e4m3_encode for whole arrays."""
    x = np.asarray(x, dtype=np.float64)
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=1e9, neginf=-1e9)), _POS[-1])
    up = np.clip(np.searchsorted(_POS, a), 1, len(_POS) - 1)     # _POS[up - 1] <= a <= _POS[up], but for a = 0
    down = up - 1
    d_up, d_down = _POS[up] - a, a - _POS[down]
    k = np.where(d_up < d_down, up, np.where(d_up > d_down, down, np.where(up % 2 == 0, up, down)))
    k = k | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isnan(x), 0x7F, k).astype(np.uint8)


def quantise_group(d32: np.ndarray):
    """d32 [T, n] float32: shift [T] and scale [T] fp16, codes [T, n] of 4 bits."""
    shift = ko.fp16_floor(d32.min(axis=1))
    low = shift.astype(np.float32)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        scale = ko.fp16_ceil((d32.max(axis=1) - low) * (np.float32(1) / np.float32(15)))
        s = scale.astype(np.float32)
        inv = np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)
        q = (d32 - low[:, None]) * inv[:, None]
    return shift, scale, np.nan_to_num(np.clip(np.rint(q), 0, 15), nan=0.0).astype(np.uint8)


def quantise(x: np.ndarray, fmt: str):
    """Rows x [..., d] (float32): (what the cache's rows hold as bytes [..., row_bytes], their scales as bytes or None)."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    lead, d = x.shape[:-1], x.shape[-1]
    if fmt == "bf16":
        return bf16_bits(x).view(np.uint8).reshape(*lead, 2 * d), None
    if fmt == "fp8":
        finite = np.where(np.isfinite(x), np.abs(x), np.float32(0))
        scale = (finite.max(-1) * (np.float32(1) / np.float32(448))).astype(np.float32)
        scale = np.where(scale < np.float32(2.0 ** -126), np.float32(0), scale)
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            inv = np.where(scale > 0, np.float32(1) / scale, np.float32(0)).astype(np.float32)
            y = np.where(np.isnan(x), x, np.where(inv[..., None] > 0, x * inv[..., None], np.float32(0)))
        return e4m3_codes(y), scale[..., None].view(np.uint8)
    g = x.reshape(-1, GROUP)
    shift, scale, codes = quantise_group(g)
    header = np.stack([shift, scale], -1).reshape(*lead, -1)
    pairs = codes.reshape(*lead, d // GROUP, GROUP // 2, 2)
    packed = pairs[..., 0] | (pairs[..., 1] << 4)                # [..., group, pair]
    return np.ascontiguousarray(np.swapaxes(packed, -1, -2)).reshape(*lead, d // 2), np.ascontiguousarray(header).view(np.uint8)


def values(rows: np.ndarray, scales, fmt: str, d: int) -> np.ndarray:
    """Float64 values [..., d] of rows and scales as bytes."""
    rows = np.ascontiguousarray(rows)
    if fmt == "bf16":
        return bf16_value(rows.view(np.uint16)).astype(np.float64)
    if fmt == "fp8":
        return kw.e4m3_decode(rows) * np.ascontiguousarray(scales).view(np.float32).astype(np.float64)
    header = np.ascontiguousarray(scales).view(np.float16).astype(np.float64).reshape(*rows.shape[:-1], d // GROUP, 2)
    out = np.empty((*rows.shape[:-1], d))
    for f in range(d):
        code = (rows[..., (f % GROUP) // 2 * (d // GROUP) + f // GROUP] >> (4 * (f % 2))) & 15
        out[..., f] = header[..., f // GROUP, 0] + header[..., f // GROUP, 1] * code
    return out


def seen(length: int, sinks: int, window: int) -> np.ndarray:
    """The tokens that the new token of a sequence attends to."""
    t = np.arange(length)
    return t if window == 0 else t[(t < sinks) | (t >= length - window)]


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One sequence and KV head: q [n, d], k and v [tokens, d] (the seen ones), all float64 -> (out [n, d], lse [n])."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(q.shape[0], -np.inf)
    s = scale * (q @ k.T)
    top = s.max(-1, keepdims=True)
    base = np.where(np.isneginf(top), 0.0, top)
    e = np.exp(s - base)
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        out = np.where(total > 0, e @ v / total, np.where(total == 0, 0.0, np.nan))
        return out, (base + np.log(total))[:, 0]


def sizes(rows: np.ndarray, scales, fmt: str, d: int) -> np.ndarray:
    """Bound of the magnitudes a value is added up from: its own, or, of 4 bits, shift and code * scale apart, a code up to 17 on the way
    (15, or of a byte's high code (whole byte - low code) / 16, up to (255 + 15) / 16)."""
    if fmt != "int4":
        return np.abs(values(rows, scales, fmt, d))
    header = np.abs(np.ascontiguousarray(scales).view(np.float16).astype(np.float64).reshape(*rows.shape[:-1], d // GROUP, 2))
    return np.repeat(header[..., 0] + 17 * header[..., 1], GROUP, axis=-1)


def attend_bound(q, k, v, k_size, v_size, scale: float, kept_bits: int, out_bits: int):
    """How far a result of fp32 arithmetic may be from attend()'s: (out [n, d], lse [n]).

    A score is a sum of d products and at most d + 16 further roundings: off by (2 d + 16) 2^-24 of the sum of their
    magnitudes.  That error, twice (numerator and denominator), the rounding of a probability to kept_bits, exponentials
    (2^-21 each) and the sums over the tokens ((n + 16) 2^-24) are relative to the sum of p |v|; the result is rounded to
    out_bits."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    n, d = k.shape
    if n == 0:
        return np.zeros_like(q), np.zeros(q.shape[0])
    s = scale * (q @ k.T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    off = (2 * d + 16) * 2.0 ** -24 * abs(scale) * (np.abs(q) @ k_size.T).max(-1)
    sums = (n + 16) * 2.0 ** -24 + 2.0 ** -20
    rel = 2 * off + 2 * sums + 2.0 ** -kept_bits
    out, lse = attend(q, k, v, scale)
    return 2.0 ** -out_bits * np.abs(out) + rel[:, None] * (p @ v_size) + 1e-37, off + sums + 2.0 ** -21 * np.abs(lse)
