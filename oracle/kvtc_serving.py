"""Places of new tokens, scaled and partial rotary positions, attention of many new tokens and joined attention on the CPU -- TEST INFRASTRUCTURE, NOT A PRODUCT PATH.

What stands between a request and the live cache of kvtc_paged.py, by the plainest definitions: one sequence, row or pair at a time, in Python's integers and in float64.  Shares no code
with the GPU library and imports nothing from it.

Readings (the paper fixes none of these):
  * free pages are taken from the end of their list, sequence after sequence; a sequence that does not fit takes none, and once the list has been asked for more than it has, no later sequence gets one;
  * frequencies scaled in bands or by a ramp divide by the factor where few turns fit the original length and not where many do;
  * a row's position is counted from the sequence's end: the last new token is the last of the sequence.

Pins (tests/test_oracle_serving.py): places worked out by hand, rotations against kvtc_rope.py, attention row by row against kvtc_paged.attend, joined halves against the whole.
"""
from __future__ import annotations

import math

import numpy as np

import kvtc_paged as kp


def place(lengths, new, page_tokens, table, free, n_tokens):
    """(starts, lengths, free pages left, slots, positions, table, lowest sequence without its place + 1 or 0)."""
    width = table.shape[1]
    table, starts, out, bad = table.copy(), [0], [], 0
    slots, positions = np.full(n_tokens, -1, np.int64), np.zeros(n_tokens, np.int32)
    taken = asked = 0
    row = 0
    for b, (had, n) in enumerate(zip(lengths, new)):
        had, n = int(had), int(n)
        first, row = row, row + max(0, n)
        starts.append(min(row, n_tokens))
        fine = had >= 0 and n >= 0 and row <= n_tokens and had + n <= min(width * page_tokens, 2 ** 31 - 1)
        if fine:
            held, need = -(-had // page_tokens), -(-(had + n) // page_tokens) - -(-had // page_tokens)
            before, asked = asked, asked + need
            fine = need == 0 or asked <= len(free)
        if not fine:
            bad = bad or b + 1
            out.append(had)
            continue
        for i in range(need):
            table[b, held + i] = free[len(free) - 1 - before - i]
        if need:
            taken = asked
        for i in range(n):
            page = int(table[b, (had + i) // page_tokens])
            slots[first + i] = page * page_tokens + (had + i) % page_tokens if page >= 0 else -1
            positions[first + i] = had + i
        out.append(had + n)
    return np.array(starts, np.int32), np.array(out, np.int32), len(free) - taken, slots, positions, table, bad


def frequencies(n, base, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0):
    """theta_j of the pairs of n rotated features."""
    if scaling == "base" and n > 2:
        base = base * factor ** (n / (n - 2))
    out = []
    for j in range(n // 2):
        theta = base ** (-2.0 * j / n)
        if scaling == "linear":
            theta /= factor
        elif scaling == "bands":
            wave = 2 * math.pi / theta
            if wave > original / low:
                theta /= factor
            elif wave > original / high:
                s = (original / wave - low) / (high - low)
                theta = (1 - s) * theta / factor + s * theta
        elif scaling == "ramp":
            pair = [n * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base)) for turns in (high, low)]
            first, last = max(0, math.floor(pair[0])), min(n - 1, math.ceil(pair[1]))
            r = (j - first) / max(last - first, 0.001)
            r = min(1.0, max(0.0, r))
            theta = (1 - r) * theta + r * theta / factor
        out.append(theta)
    return np.array(out)


def rope_scaled(x, positions, theta, pairing="half", magnitude=1.0, inverse=False):
    """x [T, heads, d] float64: the first 2 len(theta) features of every head turned."""
    x = np.asarray(x, dtype=np.float64)
    half = len(theta)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * theta[None]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    if inverse:
        c, s = c / magnitude, -s / magnitude
    else:
        c, s = c * magnitude, s * magnitude
    j = np.arange(half)
    a, b = (j, j + half) if pairing == "half" else (2 * j, 2 * j + 1)
    out = x.copy()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def seen(at: int, length: int, causal: bool, sinks: int, window: int) -> np.ndarray:
    """The tokens that a row at position `at` attends to."""
    t = np.arange(length)
    if not causal:
        return t
    t = t[t <= at]
    return t if window == 0 else t[(t < sinks) | (t > at - window)]


def served(starts, n_tokens: int):
    """Starts of any kind, [B + 1] -> the sequences that attention of many new tokens works out, and what status is: 1 + the lowest whose starts do not ascend or leave 0..n_tokens, or 0.  Left out are those, and
    what begins below a start before it (of those in 0..n_tokens), whose rows may be another's."""
    out, bad, top = [], 0, 0
    for b in range(len(starts) - 1):
        s0, s1 = int(starts[b]), int(starts[b + 1])
        if 0 <= s0 <= n_tokens:
            top = max(top, s0)
        if not 0 <= s0 <= s1 <= n_tokens:
            bad = bad or b + 1
        elif s0 == top:
            out.append(b)
    return out, bad


def bound(q, k, v, scale, key_bits, kept_bits, value_bits, out_bits):
    """kvtc_paged.attend_bound where keys, probabilities and values enter their products rounded to key_bits, kept_bits and value_bits (each off by 2^-bits of itself, at most):
    (out [n, d], lse [n])."""
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    if k.shape[0] == 0:
        return np.zeros_like(q), np.zeros(q.shape[0])
    out, lse = kp.attend_bound(q, k, v, np.abs(k), np.abs(v), scale, kept_bits, out_bits)
    s = scale * (q @ k.T)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    off = 2.0 ** -key_bits * abs(scale) * (np.abs(q) @ np.abs(k).T).max(-1)
    return out + (2 * off + 2.0 ** -value_bits)[:, None] * (p @ np.abs(v)), lse + off


def join(outs, lses):
    """Parts [rows, heads, d] and [rows, heads] -> (out, lse)."""
    lse = np.stack([np.asarray(x, dtype=np.float64) for x in lses])
    top = lse.max(0)
    base = np.where(np.isneginf(top), 0.0, top)
    with np.errstate(divide="ignore", invalid="ignore"):
        w = np.exp(lse - base)
        total = w.sum(0)
        out = sum(np.where(np.isneginf(lse[p])[..., None], 0.0, w[p][..., None] * np.asarray(outs[p], dtype=np.float64)) for p in range(len(outs)))
        return np.where(total[..., None] > 0, out / total[..., None], 0.0), base + np.log(total)
