"""Pins of the oracle of places, scaled rotations, attention of many tokens and joined attention (oracle/kvtc_serving.py)."""
import numpy as np

import kvtc_paged as kp
import kvtc_rope as kr
import kvtc_serving as sv


def test_places_worked_out_by_hand():
    table = np.array([[7, -1, -1], [3, 9, -1], [-1, -1, -1]], np.int32)
    # pages of 4: sequence 0 has 3 tokens and gets 2 (one in page 7, one in a new page), 1 has 8 and gets 1 (a new page), 2 has none and gets 5 (two pages)
    starts, lengths, left, slots, positions, out, bad = sv.place([3, 8, 0], [2, 1, 5], 4, table, [20, 21, 22, 23, 24], 9)
    assert starts.tolist() == [0, 2, 3, 8] and lengths.tolist() == [5, 9, 5] and left == 1 and bad == 0
    assert slots.tolist() == [31, 24 * 4, 23 * 4, 88, 89, 90, 91, 84, -1] and positions.tolist() == [3, 4, 8, 0, 1, 2, 3, 4, 0]
    assert out.tolist() == [[7, 24, -1], [3, 9, 23], [22, 21, -1]]


def test_a_sequence_without_place_takes_nothing():
    table = np.full((3, 2), -1, np.int32)
    starts, lengths, left, slots, positions, out, bad = sv.place([0, 0, 0], [3, 9, 2], 4, table, [5, 6], 14)      # 9 tokens are more than two pages hold
    assert bad == 2 and lengths.tolist() == [3, 0, 2] and left == 0 and starts.tolist() == [0, 3, 12, 14]
    assert slots.tolist() == [24, 25, 26] + [-1] * 9 + [20, 21] and out.tolist() == [[6, -1], [-1, -1], [5, -1]]
    # one page for two that need one each, and a third that needs none
    starts, lengths, left, slots, positions, out, bad = sv.place([0, 0, 1], [1, 1, 2], 4, np.array([[-1], [-1], [8]], np.int32), [5], 4)
    assert bad == 2 and lengths.tolist() == [1, 0, 3] and left == 0 and slots.tolist() == [20, -1, 33, 34]


def test_rotation_without_scaling_is_the_plain_one():
    rng = np.random.default_rng(1)
    x, at = rng.standard_normal((9, 3 * 16)), rng.integers(0, 5000, 9)
    for pairing in ("half", "interleaved"):
        for inverse in (False, True):
            got = sv.rope_scaled(x.reshape(9, 3, 16), at, sv.frequencies(16, 10000.0), pairing, 1.0, inverse)
            np.testing.assert_allclose(got.reshape(9, 48), kr.rope(x, at, 3, 16, 10000.0, pairing, inverse), rtol=0, atol=1e-14)
    # the first 8 features alone are heads of 8 features
    got = sv.rope_scaled(x.reshape(9, 3, 16), at, sv.frequencies(8, 10000.0))
    np.testing.assert_allclose(got[..., :8].reshape(9, 24), kr.rope(x.reshape(9, 3, 16)[..., :8].reshape(9, 24), at, 3, 8, 10000.0), rtol=0, atol=1e-14)
    np.testing.assert_array_equal(got[..., 8:], x.reshape(9, 3, 16)[..., 8:])


def test_frequencies_between_their_limits():
    plain = sv.frequencies(128, 500000.0)
    for scaling, low, high in (("bands", 1.0, 4.0), ("ramp", 1.0, 32.0)):
        f = sv.frequencies(128, 500000.0, scaling, 8.0, 8192, low, high)
        share = f / plain
        assert share[0] == 1.0 and abs(share[-1] - 1 / 8) < 1e-15 and (np.diff(share) <= 1e-15).all() and ((share > 0.2) & (share < 0.9)).any()
    np.testing.assert_allclose(sv.frequencies(128, 500000.0, "linear", 4.0), plain / 4, rtol=1e-15)
    f = sv.frequencies(128, 500000.0, "base", 4.0)                   # the slowest pair is slower by the factor, exactly
    assert f[0] == 1.0 and abs(f[-1] * 4 / plain[-1] - 1) < 1e-13
    x = np.random.default_rng(2).standard_normal((4, 2, 128))
    there = sv.rope_scaled(x, [1, 2, 3, 400], f, "half", 1.2)
    np.testing.assert_allclose(sv.rope_scaled(there, [1, 2, 3, 400], f, "half", 1.2, True), x, atol=1e-13)


def test_seen_tokens():
    assert sv.seen(3, 9, True, 0, 0).tolist() == [0, 1, 2, 3] and sv.seen(-1, 9, True, 2, 3).tolist() == []
    assert sv.seen(8, 9, True, 2, 3).tolist() == [0, 1, 6, 7, 8] and sv.seen(2, 9, True, 2, 3).tolist() == [0, 1, 2]
    assert sv.seen(3, 5, False, 0, 0).tolist() == [0, 1, 2, 3, 4]


def test_joined_halves_are_the_whole():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((5, 64)), rng.standard_normal((40, 64)), rng.standard_normal((40, 64))
    want, want_lse = kp.attend(q, k, v, 0.3)
    parts = [kp.attend(q, k[a:b], v[a:b], 0.3) for a, b in ((0, 7), (7, 7), (7, 40))]
    parts[1][0][:] = np.nan                                          # of no tokens: whatever it holds
    out, lse = sv.join([p[0][:, None] for p in parts], [p[1][:, None] for p in parts])
    np.testing.assert_allclose(out[:, 0], want, atol=1e-14)
    np.testing.assert_allclose(lse[:, 0], want_lse, atol=1e-13)
    out, lse = sv.join([np.full((1, 1, 64), np.nan)], [np.full((1, 1), -np.inf)])
    assert (out == 0).all() and np.isneginf(lse).all()
