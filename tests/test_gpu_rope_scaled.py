"""Scaled and partial rotary positions (kvtc_rope_scaled) against the float64 oracle."""
import numpy as np
import pytest
import torch

import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_gpu_cache import DEV, bits, host, to_dev

pytestmark = pytest.mark.gpu


def check(got, x, want, dtype, magnitude, where=None):
    """Sines and cosines off by 2^-24 of the magnitude, two products and a sum: a result is off by at most 4 x 2^-24 of |a| + |b| times the magnitude, and rounded to dtype once more."""
    got = got.float().cpu().numpy().astype(np.float64)
    size = 2 * np.abs(x).max(-1, keepdims=True) * max(1.0, magnitude)
    tol = 4 * 2.0 ** -24 * size + (2.0 ** -8 if dtype == kv.KVTC_BF16 else 0.0) * np.abs(want) + 1e-38
    assert (np.abs(got - want) <= tol).all(), np.abs(got - want).max()


FORMS = [("none", 1.0, 0, 0, 0), ("linear", 4.0, 0, 0, 0), ("base", 8.0, 0, 0, 0), ("bands", 8.0, 8192, 1.0, 4.0), ("ramp", 40.0, 4096, 1.0, 32.0)]
KIND = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("d,rotated,heads,beside,tokens", [(128, 128, 40, 8, 3), (128, 64, 8, 0, 700), (64, 16, 3, 1, 257), (80, 20, 5, 0, 33), (96, 24, 2, 3, 130), (256, 256, 1, 0, 65), (256, 64, 2, 2, 9),
                                                          (2, 2, 7, 1, 50), (6, 4, 3, 0, 50), (128, 126, 2, 0, 17), (64, 64, 1, 0, 1), (128, 2, 1, 0, 1000)])
def test_rotations_are_the_oracles(dtype, pairing, d, rotated, heads, beside, tokens):
    rng = np.random.default_rng(d + rotated + tokens)
    scaling, factor, original, low, high = FORMS[(d + rotated + heads + tokens) % 5]
    magnitude = 1.0 if scaling != "ramp" else 1.3689
    form = kv.rope_form(rotated, kv.ROPE_HALF if pairing == "half" else kv.ROPE_INTERLEAVED, 500000.0, KIND[scaling], factor, original, low, high, magnitude)
    theta = sv.frequencies(rotated, 500000.0, scaling, factor, original, low, high)
    x = host(rng.standard_normal((tokens, heads + beside, d)).astype(np.float32) * 3, dtype)
    xd = to_dev(x, dtype)
    at = rng.integers(-5, 1_000_000, tokens).astype(np.int32)
    at[0] = 2 ** 31 - 1
    wide = (heads + beside) * d
    for inverse, positions in ((False, at), (True, None)):
        want = sv.rope_scaled(x[:, :heads], at if positions is not None else np.arange(131000, 131000 + tokens), theta, pairing, magnitude, inverse)
        out = torch.full((tokens + 1, heads, d), 5.0, dtype=xd.dtype, device=DEV)
        kv.kvtc_rope_scaled(xd, out, dtype, tokens, heads, d, wide, d, heads * d, d, torch.from_numpy(positions).to(DEV) if positions is not None else None, 131000, form, inverse)
        torch.cuda.synchronize()
        check(out[:tokens], x[:, :heads], want, dtype, magnitude)
        np.testing.assert_array_equal(bits(out[:tokens, :, rotated:]), bits(xd[:, :heads, rotated:].contiguous()))
        assert bool((out[tokens] == 5.0).all())
        # in place, inside the fused row: the same; what stands beside stays
        both = xd.clone()
        kv.kvtc_rope_scaled(both, both, dtype, tokens, heads, d, wide, d, wide, d, torch.from_numpy(positions).to(DEV) if positions is not None else None, 131000, form, inverse)
        torch.cuda.synchronize()
        assert torch.equal(both[:, :heads], out[:tokens]) and torch.equal(both[:, heads:], xd[:, heads:])


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_heads_first_and_odd_strides(dtype):
    """From a heads-first tensor into a token-major one and back, from addresses and strides that allow no wide pieces."""
    rng = np.random.default_rng(3)
    tokens, heads, d = 333, 4, 64
    form, theta = kv.rope_form(32, kv.ROPE_HALF, 10000.0), sv.frequencies(32, 10000.0)
    x = host(rng.standard_normal((tokens, heads, d)).astype(np.float32), dtype)
    want = sv.rope_scaled(x, np.arange(-7, tokens - 7), theta)
    first = to_dev(np.ascontiguousarray(x.transpose(1, 0, 2)), dtype)
    out = torch.empty((tokens, heads, d), dtype=first.dtype, device=DEV)
    kv.kvtc_rope_scaled(first, out, dtype, tokens, heads, d, d, tokens * d, heads * d, d, None, -7, form)
    torch.cuda.synchronize()
    check(out, x, want, dtype, 1.0)
    for gap, shift in ((1, 1), (2, 3), (4, 0), (8, 4)):
        head, row = d + gap, heads * (d + gap) + gap
        flat = torch.full((tokens * row + 64,), 7.0, dtype=first.dtype, device=DEV)
        at = (torch.arange(tokens)[:, None, None] * row + torch.arange(heads)[None, :, None] * head + torch.arange(d)).to(DEV) + shift
        kv.kvtc_rope_scaled(first, flat.data_ptr() + shift * flat.element_size(), dtype, tokens, heads, d, d, tokens * d, row, head, None, -7, form)
        torch.cuda.synchronize()
        assert torch.equal(flat[at], out)
        flat[at] = 7.0
        assert bool((flat == 7.0).all())
        back = torch.empty_like(first)
        flat[at] = out
        kv.kvtc_rope_scaled(flat.data_ptr() + shift * flat.element_size(), back, dtype, tokens, heads, d, row, head, d, tokens * d, None, -7, form, True)
        torch.cuda.synchronize()
        got = out.float().cpu().numpy()
        check(back.transpose(0, 1), got, sv.rope_scaled(got, np.arange(-7, tokens - 7), theta, inverse=True), dtype, 1.0)


def test_zero_angles_and_special_values():
    form = kv.rope_form(64, kv.ROPE_HALF, 10000.0)
    x = torch.randn((2, 3, 64), device=DEV)
    x[1, 0, 3], x[1, 1, 40], x[1, 2, 5] = float("inf"), float("nan"), -0.0
    out = torch.empty_like(x)
    kv.kvtc_rope_scaled(x, out, kv.KVTC_F32, 2, 3, 64, 192, 64, 192, 64, torch.tensor([0, 9], dtype=torch.int32, device=DEV), 0, form)
    torch.cuda.synchronize()
    assert torch.equal(out[0], x[0])                                 # position 0 turns nothing
    assert bool(torch.isinf(out[1, 0, [3, 35]]).all()) and bool(torch.isnan(out[1, 1, [8, 40]]).all()) and int((~torch.isfinite(out)).sum()) == 4


def test_many_tokens_and_far_positions():
    """More than one unit to a thread and a workgroup, positions whose angles are reduced and ones beyond that."""
    rng = np.random.default_rng(4)
    tokens = 5001
    x = rng.standard_normal((tokens, 2, 64)).astype(np.float32)
    at = rng.integers(-2 ** 31, 2 ** 31, tokens).astype(np.int32)
    form = kv.rope_form(64, kv.ROPE_INTERLEAVED, 0.5)                # frequencies above 1: angles beyond 2^31
    out = torch.empty((tokens, 2, 64), device=DEV)
    kv.kvtc_rope_scaled(to_dev(x, kv.KVTC_F32), out, kv.KVTC_F32, tokens, 2, 64, 128, 64, 128, 64, torch.from_numpy(at).to(DEV), 0, form)
    torch.cuda.synchronize()
    check(out, x, sv.rope_scaled(x, at, np.array(form.theta[:32]), "interleaved"), kv.KVTC_F32, 1.0)
