"""The live cache's entry points on the CPU: sizes, the descriptor's layout, and every argument error, found before any launch."""
import ctypes as C

import pytest

import paper_2511_01815_amd as kv

SMALL, ARG, UNSUPPORTED = 3, 1, 2


def _cache(**change):
    """A valid descriptor over addresses that are never touched: 4 heads of 128, pages [heads][16 tokens] in 8 bits."""
    row = 128
    d = dict(format=kv.KVTC_CACHE_FP8, n_pages=10, page_tokens=16, n_heads=4, d_head=128, k_dev=1 << 20, v_dev=2 << 20, page_stride=4 * 16 * row,
             head_stride=16 * row, token_stride=row, k_scales_dev=3 << 20, v_scales_dev=4 << 20)
    d.update(change)
    return kv.cache(**d)


def _write(cache, k=1 << 24, v=1 << 25, dtype=0, n=5, ts=512, hs=128, slots=1 << 26, status=None):
    return kv.lib().kvtc_cache_write(C.byref(cache) if cache is not None else None, k, v, dtype, n, ts, hs, slots, status, None)


def _read(cache, k=1 << 24, v=1 << 25, dtype=0, n=5, ts=512, hs=128, slots=1 << 26, status=None):
    return kv.lib().kvtc_cache_read(C.byref(cache) if cache is not None else None, slots, n, k, v, dtype, ts, hs, status, None)


def _attend(cache, q=1 << 24, dtype=0, n=3, hq=8, qs=1024, qh=128, pages=1 << 26, ps=7, lengths=1 << 27, most=100, scale=0.1, sinks=0, window=0, out=1 << 28,
            lse=None, work=1 << 29, nbytes=1 << 40, status=None):
    return kv.lib().kvtc_attend(C.byref(cache) if cache is not None else None, q, dtype, n, hq, qs, qh, pages, ps, lengths, most, scale, sinks, window, out, lse,
                                work, nbytes, status, None)


def test_descriptor_layout_and_sizes():
    assert C.sizeof(kv.KvtcCache) == 16 + 4 * 8 + 4 * 8
    assert kv.KvtcCache.n_pages.offset == 16 and kv.KvtcCache.k_dev.offset == 48 and kv.KvtcCache.v_scales_dev.offset == 72
    for d in (64, 128, 256):
        assert [kv.kvtc_cache_row_bytes(f, d) for f in range(3)] == [2 * d, d, d // 2]
        assert [kv.kvtc_cache_scale_bytes(f, d) for f in range(3)] == [0, 4, d // 8]
    for f, d in ((0, 96), (3, 128), (-1, 128), (1, 0), (2, 512)):
        assert kv.kvtc_cache_row_bytes(f, d) == 0 and kv.kvtc_cache_scale_bytes(f, d) == 0


def test_nothing_to_do_is_no_error():
    assert _write(_cache(), k=None, v=None, slots=None, n=0) == 0
    assert _read(_cache(), k=None, v=None, slots=None, n=0) == 0
    assert _attend(_cache(), q=None, pages=None, lengths=None, out=None, work=None, n=0) == 0


BAD_CACHES = [
    (dict(format=3), ARG), (dict(format=-1), ARG), (dict(d_head=96), UNSUPPORTED), (dict(d_head=0), UNSUPPORTED), (dict(n_heads=0), ARG), (dict(n_heads=1025), ARG),
    (dict(page_tokens=0), ARG), (dict(n_pages=0), ARG), (dict(n_pages=1 << 31), ARG), (dict(k_dev=None), ARG), (dict(v_dev=None), ARG),
    (dict(k_dev=(1 << 20) + 8), ARG), (dict(token_stride=136), ARG), (dict(page_stride=8192 + 8), ARG),
    (dict(token_stride=112), ARG),                               # a row runs into the next token's
    (dict(head_stride=15 * 128), ARG),                           # a head's tokens run into the next head's
    (dict(page_stride=4 * 16 * 128 - 16), ARG), (dict(token_stride=-128), ARG), (dict(head_stride=0), ARG),
    (dict(k_scales_dev=None), ARG), (dict(v_scales_dev=None), ARG), (dict(v_scales_dev=(4 << 20) + 4), ARG),
    (dict(page_tokens=1 << 24, token_stride=1 << 8, head_stride=1 << 32, page_stride=1 << 36), ARG),      # a page's tokens over 2^31 bytes
    (dict(page_stride=1 << 62, n_pages=1 << 20), ARG),           # the pool passes 63 bits
]


@pytest.mark.parametrize("change,want", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(change, want):
    c = _cache(**change)
    assert _write(c) == want and "kvtc_cache_write" in kv.kvtc_last_error()
    assert _read(c) == want and "kvtc_cache_read" in kv.kvtc_last_error()
    assert _attend(c) == want and "kvtc_attend" in kv.kvtc_last_error()
    assert kv.kvtc_attend_work_bytes(c, 3, 8, 100) == 0


def test_no_cache_at_all():
    assert _write(None) == ARG and _read(None) == ARG and _attend(None) == ARG


@pytest.mark.parametrize("call", [_write, _read])
def test_bad_tokens_are_refused(call):
    c = _cache()
    assert call(c, n=-1) == ARG and call(c, n=1 << 31) == ARG
    assert call(c, dtype=2) == ARG
    assert call(c, k=None) == ARG and call(c, v=None) == ARG and call(c, slots=None) == ARG
    assert call(c, k=(1 << 24) + 2) == ARG and call(c, slots=(1 << 26) + 4) == ARG and call(c, status=(1 << 27) + 2) == ARG
    assert call(c, ts=516) == ARG and call(c, hs=132, ts=1024) == ARG          # not 16-byte aligned
    assert call(c, ts=504) == ARG                                              # a token's heads run into the next token
    assert call(c, ts=128, hs=4 * 128) == ARG                                  # heads-major, a head's slab shorter than its tokens
    assert call(c, ts=-512) == ARG
    assert "overlap" in kv.kvtc_last_error()


def test_bad_attention_is_refused():
    c = _cache()
    assert _attend(c, n=-1) == ARG and _attend(c, n=65537) == ARG
    assert _attend(c, hq=0) == ARG and _attend(c, hq=6) == ARG and _attend(c, hq=1028) == ARG
    assert _attend(c, most=0) == ARG and _attend(c, most=1 << 31) == ARG
    assert _attend(c, n=65536, most=1 << 23, ps=1 << 30) == UNSUPPORTED        # more tiles than 31 bits count
    assert _attend(c, dtype=2) == ARG
    for name in ("q", "pages", "lengths", "out", "work"):
        assert _attend(c, **{name: None}) == ARG and "null" in kv.kvtc_last_error()
    assert _attend(c, q=(1 << 24) + 8) == ARG and _attend(c, qs=1028) == ARG and _attend(c, qh=130) == ARG and _attend(c, qs=-1024) == ARG
    assert _attend(c, out=(1 << 28) + 8) == ARG and _attend(c, lse=(1 << 30) + 2) == ARG and _attend(c, work=(1 << 29) + 128) == ARG
    assert _attend(c, pages=(1 << 26) + 2) == ARG and _attend(c, lengths=(1 << 27) + 1) == ARG and _attend(c, status=(1 << 30) + 1) == ARG
    assert _attend(c, ps=6) == ARG                                             # 6 pages of 16 tokens for 100
    assert _attend(c, scale=float("nan")) == ARG and _attend(c, scale=float("inf")) == ARG
    assert _attend(c, sinks=-1) == ARG and _attend(c, window=-1) == ARG
    need = kv.kvtc_attend_work_bytes(c, 3, 8, 100)
    assert need > 0 and _attend(c, nbytes=need - 1) == SMALL
    for n, hq, most in ((-1, 8, 100), (3, 7, 100), (3, 8, 0)):
        assert kv.kvtc_attend_work_bytes(c, n, hq, most) == 0


def test_strides_may_nest_in_any_order():
    """Descriptors that are valid (refused only for the workspace that is too small, the last check)."""
    row, page, heads, pages = 128, 16, 4, 10
    for token, head, pstride in ((row, row * page, row * page * heads), (row * heads, row, row * page * heads), (row, row * page * pages, row * page),
                                 (row * heads * pages, row, row * heads), (row * heads, row * heads * page * pages, row * heads * page)):
        assert _attend(_cache(token_stride=token, head_stride=head, page_stride=pstride), nbytes=0) == SMALL
    assert _attend(_cache(n_pages=1, page_stride=0), nbytes=0) == SMALL                         # one page: no stride to speak of
    assert _attend(_cache(format=kv.KVTC_CACHE_INT4, k_scales_dev=1 << 10, token_stride=64), nbytes=0) == SMALL
    assert _attend(_cache(format=kv.KVTC_CACHE_BF16, k_scales_dev=None, v_scales_dev=None, token_stride=256, head_stride=4096, page_stride=16384), nbytes=0) == SMALL


def test_errors_are_raised_by_the_binding():
    with pytest.raises(kv.KvtcError, match="KVTC_E_UNSUPPORTED"):
        kv.kvtc_cache_write(_cache(d_head=80), 16, 16, kv.KVTC_BF16, 1, 512, 128, 16, None, 0)
