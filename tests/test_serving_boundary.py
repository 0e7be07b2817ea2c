"""Places, scaled rotations, attention of many new tokens and joined attention on the CPU: sizes, layouts of descriptors, and every argument error, found before any launch."""
import ctypes as C
import math

import numpy as np
import pytest

import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_cache_boundary import ARG, BAD_CACHES, SMALL, UNSUPPORTED, _cache


def _place(n=3, lengths=1 << 20, new=2 << 20, page=16, pages=3 << 20, ps=7, free=4 << 20, n_free=5 << 20, rows=10, starts=6 << 20, out=7 << 20, left=8 << 20, slots=9 << 20, at=10 << 20, status=None):
    return kv.lib().kvtc_cache_place(n, lengths, new, page, pages, ps, free, n_free, rows, starts, out, left, slots, at, status, None)


def test_bad_places_are_refused():
    assert _place(n=-1) == ARG and _place(n=65537) == ARG and _place(rows=-1) == ARG and _place(rows=1 << 31) == ARG
    assert _place(page=0) == ARG and _place(ps=0) == ARG and _place(ps=1 << 31) == ARG
    for name in ("lengths", "new", "pages", "free", "n_free", "starts", "out", "left", "slots"):
        assert _place(**{name: None}) == ARG and "null" in kv.kvtc_last_error(), name
        assert _place(**{name: (1 << 20) + 2}) == ARG and "misaligned" in kv.kvtc_last_error(), name
    assert _place(slots=(1 << 20) + 4) == ARG and _place(at=(1 << 20) + 1) == ARG and _place(status=6) == ARG


def _rope(form, x=1 << 20, out=1 << 21, dtype=0, n=5, h=4, d=128, ts=512, hs=128, ots=512, ohs=128, at=None, first=0, inverse=0):
    return kv.lib().kvtc_rope_scaled(x, out, dtype, n, h, d, ts, hs, ots, ohs, at, first, C.byref(form) if form is not None else None, inverse, None)


def test_bad_rotations_are_refused():
    f = kv.rope_form(64, kv.ROPE_HALF, 10000.0)
    assert _rope(None) == ARG and _rope(kv.KvtcRopeForm()) == ARG                # not made by kvtc_rope_form_init
    assert _rope(kv.rope_form(130, kv.ROPE_HALF, 10000.0)) == ARG               # more than the head has
    assert _rope(f, n=-1) == ARG and _rope(f, n=1 << 31) == ARG and _rope(f, h=0) == ARG and _rope(f, h=1025) == ARG and _rope(f, d=129) == ARG and _rope(f, d=258) == ARG
    assert _rope(f, dtype=2) == ARG and _rope(f, inverse=2) == ARG and _rope(f, x=None) == ARG and _rope(f, out=None) == ARG
    assert _rope(f, x=(1 << 20) + 1) == ARG and _rope(f, out=(1 << 21) + 2, dtype=1) == ARG and _rope(f, at=(1 << 22) + 2) == ARG
    assert _rope(f, ts=508) == ARG and _rope(f, ohs=120) == ARG and _rope(f, ots=-512) == ARG and _rope(f, ts=128, hs=4 * 128) == ARG
    assert "overlap" in kv.kvtc_last_error()
    assert _rope(f, out=1 << 20, ots=1024) == ARG and "in place" in kv.kvtc_last_error()
    assert _rope(f, first=(1 << 62) + 1) == ARG and _rope(f, first=-(1 << 62) - 1) == ARG
    assert _rope(f, first=(1 << 62) + 1) == ARG and _rope(f, first=-(1 << 62) - 1) == ARG
    assert _rope(f, n=0, x=None, out=None) == 0


@pytest.mark.parametrize("n,pairing,base,scaling,factor,original,low,high,magnitude", [
    (0, 0, 1e4, 0, 1, 0, 0, 0, 1), (63, 0, 1e4, 0, 1, 0, 0, 0, 1), (258, 0, 1e4, 0, 1, 0, 0, 0, 1), (64, 2, 1e4, 0, 1, 0, 0, 0, 1), (64, 0, 0.0, 0, 1, 0, 0, 0, 1),
    (64, 0, math.inf, 0, 1, 0, 0, 0, 1), (64, 0, 1e4, 5, 1, 0, 0, 0, 1), (64, 0, 1e4, 1, 0.0, 0, 0, 0, 1), (64, 0, 1e4, 2, math.nan, 0, 0, 0, 1), (64, 0, 1e4, 3, 8, 0, 1, 4, 1),
    (64, 0, 1e4, 3, 8, 8192, 4, 4, 1), (64, 0, 1e4, 4, 8, 8192, 0, 4, 1), (64, 0, 1.0, 4, 8, 8192, 1, 32, 1), (64, 0, 1e4, 0, 1, 0, 0, 0, 0.0), (64, 0, 1e4, 0, 1, 0, 0, 0, 1e39),
    (64, 0, 1e4, 0, 1, 0, 0, 0, -1.0), (64, 0, 1e4, 0, 1, 0, 0, 0, 1e-46)])
def test_bad_forms_are_refused(n, pairing, base, scaling, factor, original, low, high, magnitude):
    with pytest.raises(kv.KvtcError, match="KVTC_E_ARG"):
        kv.rope_form(n, pairing, base, scaling, factor, original, low, high, magnitude)


@pytest.mark.parametrize("n", [2, 20, 64, 128, 256])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands", "ramp"])
def test_forms_hold_the_oracles_frequencies(n, scaling):
    kind = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}[scaling]
    for factor, original, low, high in ((1.0, 4096, 1, 4), (8.0, 8192, 1, 4), (40.0, 2048, 1, 32), (0.5, 300, 0.1, 7)):
        f = kv.rope_form(n, kv.ROPE_HALF, 500000.0, kind, factor, original, low, high, 1.25)
        assert f.n_rotated == n and f.magnitude == 1.25 and list(f.theta[n // 2:]) == [0.0] * (128 - n // 2)
        np.testing.assert_allclose(f.theta[:n // 2], sv.frequencies(n, 500000.0, scaling, factor, original, low, high), rtol=1e-13)       # (a few roundings, and pow's)
    assert C.sizeof(kv.KvtcRopeForm) == 16 + 8 * 128


def _many(cache, q=1 << 24, dtype=0, n=3, rows=20, hq=8, qs=1024, qh=128, starts=1 << 25, pages=1 << 26, ps=7, lengths=1 << 27, most=100, scale=0.1, causal=1, sinks=0, window=0, out=1 << 28,
          lse=None, work=1 << 29, nbytes=1 << 40, status=None):
    return kv.lib().kvtc_attend_many(C.byref(cache) if cache is not None else None, q, dtype, n, rows, hq, qs, qh, starts, pages, ps, lengths, most, scale, causal, sinks, window, out, lse, work,
                                     nbytes, status, None)


@pytest.mark.parametrize("change,want", BAD_CACHES)
def test_bad_caches_are_refused(change, want):
    c = _cache(**change)
    assert _many(c) == want and "kvtc_attend_many" in kv.kvtc_last_error()
    assert kv.kvtc_attend_many_work_bytes(c, 3, 20, 8, 100) == 0


def test_bad_attention_is_refused():
    c = _cache()
    assert _many(None) == ARG
    assert _many(c, n=-1) == ARG and _many(c, n=65537) == ARG and _many(c, rows=-1) == ARG and _many(c, rows=1 << 31) == ARG
    assert _many(c, hq=0) == ARG and _many(c, hq=6) == ARG and _many(c, hq=1028) == ARG
    assert _many(c, rows=(1 << 27) + 1) == UNSUPPORTED                           # more than 2^30 rows
    assert _many(c, most=0) == ARG and _many(c, most=1 << 31) == ARG and _many(c, dtype=2) == ARG
    for name in ("q", "starts", "pages", "lengths", "out", "work"):
        assert _many(c, **{name: None}) == ARG and "null" in kv.kvtc_last_error()
    assert _many(c, q=(1 << 24) + 8) == ARG and _many(c, qs=1028) == ARG and _many(c, qh=130) == ARG and _many(c, qs=-1024) == ARG and _many(c, qh=1 << 41) == ARG
    assert _many(c, out=(1 << 28) + 8) == ARG and _many(c, lse=(1 << 30) + 2) == ARG and _many(c, work=(1 << 29) + 128) == ARG
    assert _many(c, starts=(1 << 25) + 2) == ARG and _many(c, pages=(1 << 26) + 2) == ARG and _many(c, lengths=(1 << 27) + 1) == ARG and _many(c, status=(1 << 30) + 1) == ARG
    assert _many(c, ps=6) == ARG                                                 # 6 pages of 16 tokens for 100
    assert _many(c, scale=float("nan")) == ARG and _many(c, scale=float("inf")) == ARG
    assert _many(c, causal=2) == ARG and _many(c, sinks=-1) == ARG and _many(c, window=-1) == ARG and _many(c, causal=0, window=5) == ARG
    need = kv.kvtc_attend_many_work_bytes(c, 3, 20, 8, 100)
    assert need > 0 and _many(c, nbytes=need - 1) == SMALL
    for n, rows, hq, most in ((-1, 20, 8, 100), (3, -1, 8, 100), (3, 20, 7, 100), (3, 20, 8, 0)):
        assert kv.kvtc_attend_many_work_bytes(c, n, rows, hq, most) == 0
    assert _many(c, n=0, q=None, out=None, work=None, nbytes=0) == 0 and _many(c, rows=0, q=None, out=None, work=None, nbytes=0) == 0


def _join(n=2, outs=(1 << 20, 1 << 21), lses=(1 << 22, 1 << 23), dtype=0, rows=5, heads=4, d=128, out=1 << 24, out_dtype=0, lse=None):
    a, b = (C.c_void_p * len(outs))(*outs), (C.c_void_p * len(lses))(*lses)
    return kv.lib().kvtc_attend_join(n, a, b, dtype, rows, heads, d, out, out_dtype, lse, None)


def test_bad_joins_are_refused():
    assert _join(n=0) == ARG and _join(n=17, outs=[1 << 20] * 17, lses=[1 << 22] * 17) == ARG
    assert _join(dtype=2) == ARG and _join(out_dtype=-1) == ARG and _join(rows=-1) == ARG and _join(rows=1 << 31) == ARG and _join(heads=0) == ARG and _join(heads=1025) == ARG
    assert _join(d=96) == UNSUPPORTED and _join(out=None) == ARG and _join(outs=(1 << 20, None)) == ARG and _join(lses=(None, 1 << 22)) == ARG
    assert _join(outs=(1 << 20, (1 << 21) + 8)) == ARG and _join(lses=(1 << 22, (1 << 23) + 2)) == ARG and _join(out=(1 << 24) + 8) == ARG and _join(lse=(1 << 25) + 1) == ARG
    assert _join(out=1 << 21, out_dtype=1) == ARG                                # a part's place in another type
    assert kv.lib().kvtc_attend_join(2, None, None, 0, 5, 4, 128, 1 << 24, 0, None, None) == ARG
    assert _join(rows=0, outs=(None, None), lses=(None, None), out=None) == 0
    with pytest.raises(ValueError):
        kv.kvtc_attend_join([16], [16, 32], 0, 1, 1, 64, 16, 0, None, 0)
