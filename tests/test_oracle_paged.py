"""Pins of the live cache's oracle (CPU only)."""
import numpy as np
import pytest

import kvtc_oracle as ko
import kvtc_paged as kp
import kvtc_window as kw


def test_e4m3_codes_are_the_sinks_oracles():
    rng = np.random.default_rng(1)
    t = kw.e4m3_table()[:0x7F]
    x = np.concatenate([rng.standard_normal(400) * np.exp(rng.normal(0, 4, 400)), t, -t, (t[1:] + t[:-1]) / 2, [np.inf, -np.inf, np.nan, 0.0, -0.0, 449, 1e30]])
    np.testing.assert_array_equal(kp.e4m3_codes(x), kw.e4m3_encode(x))


def test_bf16_rounding_is_the_coders():
    rng = np.random.default_rng(2)
    x = (rng.standard_normal(5000) * np.exp(rng.normal(0, 8, 5000))).astype(np.float32)
    x[:3] = [1 + 2.0 ** -9, 1 + 3 * 2.0 ** -9, -2.0 ** -130]
    np.testing.assert_array_equal(kp.bf16_value(kp.bf16_bits(x)), ko.bf16_round(x))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("fmt,most", [("bf16", 2.0 ** -8), ("fp8", 2.0 ** -4), ("int4", None)])
def test_values_are_near_what_was_quantised(d, fmt, most):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((7, 3, d)).astype(np.float32) * 3
    rows, scales = kp.quantise(x, fmt)
    assert rows.shape == (7, 3, {"bf16": 2 * d, "fp8": d, "int4": d // 2}[fmt]) and rows.dtype == np.uint8
    got = kp.values(rows, scales, fmt, d)
    if fmt == "int4":                                            # half a step of the group, and the header's rounding
        g = x.reshape(7, 3, d // 32, 32)
        step = (g.max(-1) - g.min(-1)) / 15
        assert (np.abs(got - x).reshape(g.shape) <= 0.51 * step[..., None] + 0.01).all()
    else:
        top = np.abs(x).max(-1, keepdims=True) if fmt == "fp8" else 0
        assert (np.abs(got - x) <= most * np.abs(x) + 2.0 ** -9 * top / 448 * 1.01).all()


def test_groups_of_four_bits_are_the_coders_but_for_a_last_place_of_the_scale():
    """A range times 1 / 15 in float32 is within one place of the range divided by 15, so a scale is the coder's or its neighbour, and rarely that."""
    rng = np.random.default_rng(6)
    g = (rng.standard_normal((20000, 32)) * np.exp(rng.normal(0, 3, (20000, 1)))).astype(np.float32)
    shift, scale, codes = kp.quantise_group(g)
    want = ko.quantise_group(g, 4)
    np.testing.assert_array_equal(shift.view(np.uint16), want[0].view(np.uint16))
    apart = np.abs(scale.view(np.uint16).astype(int) - want[1].view(np.uint16).astype(int))
    assert apart.max() <= 1 and apart.mean() < 0.01
    same = apart == 0
    np.testing.assert_array_equal(codes[same], want[2][same])


def test_a_row_of_four_bits_packed_by_hand():
    """64 features: 0 .. 15 four times over in the first group's order, the second group reversed: shift 0, scale 1, code = value."""
    x = np.concatenate([np.arange(32) % 16, 15 - np.arange(32) % 16]).astype(np.float32)[None]
    rows, scales = kp.quantise(x, "int4")
    np.testing.assert_array_equal(scales.view(np.float16).reshape(2, 2), [[0, 1], [0, 1]])
    for pair in range(16):
        for group in range(2):
            a, b = int(x[0, group * 32 + 2 * pair]), int(x[0, group * 32 + 2 * pair + 1])
            assert rows[0, pair * 2 + group] == a | b << 4
    np.testing.assert_array_equal(kp.values(rows, scales, "int4", 64), x)


def test_rows_that_are_zero_tiny_or_not_finite():
    x = np.zeros((4, 64), np.float32)
    x[1] = 1e-37                                                 # 1e-37 / 448 is below the smallest normal number
    x[2, 0], x[2, 1], x[2, 2], x[2, 3] = np.inf, -np.inf, np.nan, 7.0
    x[3] = -3.0
    rows, scales = kp.quantise(x, "fp8")
    got = kp.values(rows, scales, "fp8", 64)
    near = lambda v, want: np.abs(v - want) <= 2.0 ** -22 * abs(want)          # (1 / 448 and the scale are each rounded to float32)
    assert (got[:2] == 0).all() and near(got[3], -3.0).all()
    assert near(got[2, 0], 7.0) and near(got[2, 1], -7.0) and np.isnan(got[2, 2]) and near(got[2, 3], 7.0) and (got[2, 4:] == 0).all()


def test_attention_in_closed_form():
    rng = np.random.default_rng(4)
    v = rng.standard_normal((6, 8))
    q = rng.standard_normal((2, 8))
    out, lse = kp.attend(q, np.zeros((6, 8)), v, 0.5)            # equal scores: the mean
    np.testing.assert_allclose(out, np.broadcast_to(v.mean(0), (2, 8)), rtol=1e-14)
    np.testing.assert_allclose(lse, np.log(6.0), rtol=1e-14)
    k = rng.standard_normal((6, 8))
    out, lse = kp.attend(q, k[:1], v[:1], 0.5)                   # one token: its value
    np.testing.assert_allclose(out, np.broadcast_to(v[0], (2, 8)), rtol=1e-14)
    np.testing.assert_allclose(lse, 0.5 * (q @ k[0]), rtol=1e-14)
    out, lse = kp.attend(q, k[:0], v[:0], 0.5)
    assert (out == 0).all() and np.isneginf(lse).all()
    whole = kp.attend(q, k, v, 0.5)                              # two parts joined by their sums
    a, b = kp.attend(q, k[:2], v[:2], 0.5), kp.attend(q, k[2:], v[2:], 0.5)
    wa = 1 / (1 + np.exp(b[1] - a[1]))[:, None]
    np.testing.assert_allclose(whole[0], wa * a[0] + (1 - wa) * b[0], rtol=1e-12)
    np.testing.assert_allclose(whole[1], np.logaddexp(a[1], b[1]), rtol=1e-12)


def test_what_a_window_sees():
    assert kp.seen(5, 0, 0).tolist() == [0, 1, 2, 3, 4]
    assert kp.seen(9, 2, 3).tolist() == [0, 1, 6, 7, 8]
    assert kp.seen(4, 2, 3).tolist() == [0, 1, 2, 3]
    assert kp.seen(3, 7, 1).tolist() == [0, 1, 2]
    assert kp.seen(0, 4, 4).tolist() == []


def test_the_bound_holds_for_fp32_arithmetic_and_is_not_loose_for_one_part():
    """attend() again with every step in float32 stays inside; probabilities rounded to bf16 alone do not."""
    rng = np.random.default_rng(5)
    q, k, v = (rng.standard_normal(s).astype(np.float32) for s in ((3, 64), (500, 64), (500, 64)))
    want, want_lse = kp.attend(q, k, v, 0.125)
    tol, tol_lse = kp.attend_bound(q, k, v, np.abs(k), np.abs(v), 0.125, 24, 24)
    s = (np.float32(0.125) * (q @ k.T)).astype(np.float32)
    e = np.exp(s - s.max(-1, keepdims=True)).astype(np.float32)
    got = (e @ v) / e.sum(-1, keepdims=True)
    assert (np.abs(got - want) <= tol).all()
    assert (np.abs(s.max(-1) + np.log(e.sum(-1)) - want_lse) <= tol_lse).all()
    one = (ko.bf16_round(e) @ v) / e.sum(-1, keepdims=True)
    assert (np.abs(one - want) > tol).any()
