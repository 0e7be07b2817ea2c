"""By which kernel, and in how many parts, a kvtc_attend_many runs, on the CPU: the rules are the host's."""
import ctypes as C

import pytest

import paper_2511_01815_amd as kv
from test_attend_route import FORMATS, cache_of


def route(cache, dtype, n_seqs, n_tokens, n_q_heads, max_tokens, sinks=0, window=0):
    got = (C.c_int32 * 6)()
    assert kv.lib().kvtc_host_attend_many_route(C.byref(cache), dtype, n_seqs, n_tokens, n_q_heads, max_tokens, sinks, window, got) == 0, kv.kvtc_last_error()
    return dict(zip(("kind", "rows", "tile", "items", "parts", "part_tiles"), got))


def most_tiles(r, group, max_tokens, sinks, window):
    """Tiles of an item, at most: of all its sequence's tokens, or of the sinks and of what its rows see behind them."""
    every = -(-max_tokens // r["tile"])
    if window == 0:
        return every
    span = min(window, max_tokens) + -(-r["rows"] // group)       # tokens that some row of an item sees in its window
    return min(every, -(-min(sinks, max_tokens) // r["tile"]) + (span + r["tile"] - 2) // r["tile"] + 1)


SIZES = [(n, t, m) for n in (1, 2, 7, 64, 4096, 65536) for t in (1, 3, 33, 200, 5000, 1 << 20) for m in (1, 20, 700, 5000, 40000, 1 << 20, 2 ** 31 - 1)]


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,group", [(1, 1), (8, 4), (2, 24), (1, 1024)])
def test_parts_cover_every_tile_and_fit_the_workspace(fmt, d, heads, group):
    cache, seen, accepted = cache_of(fmt, heads, d, 64), set(), 0
    for n_seqs, each, max_tokens in SIZES:
        n_tokens, hq = n_seqs * each, heads * group
        if n_tokens * hq > 1 << 29:
            if n_tokens < 1 << 31:
                assert kv.kvtc_attend_many_work_bytes(cache, n_seqs, n_tokens, hq, max_tokens) == 0
            continue
        work = kv.kvtc_attend_many_work_bytes(cache, n_seqs, n_tokens, hq, max_tokens)
        for dtype in (kv.KVTC_BF16, kv.KVTC_F32):
            for sinks, window in ((0, 0), (0, 1), (4, 128), (1000, 3000), (7, 1 << 40)):
                r = route(cache, dtype, n_seqs, n_tokens, hq, max_tokens, sinks, window)
                assert (r["kind"] == 0) == (dtype == kv.KVTC_F32) and r["rows"] in (32, 64, 128)
                assert r["items"] == n_tokens * group // r["rows"] + n_seqs and r["items"] * 256 < 1 << 32
                assert 1 <= r["parts"] <= 512
                if r["parts"] > 1:
                    assert r["parts"] * r["part_tiles"] >= most_tiles(r, group, max_tokens, sinks, window), (n_seqs, each, max_tokens, sinks, window, r)
                    assert r["parts"] * n_tokens * hq * (d + 2) * 4 <= work
                seen.add((r["kind"], r["parts"] > 1))
                accepted += 1
    assert accepted > 200 and (0, True) in seen and (0, False) in seen


def test_refusals_of_the_route():
    c = cache_of("fp8", 4, 64, 16)
    f, got = kv.lib().kvtc_host_attend_many_route, (C.c_int32 * 6)()
    bad = [(0, 0, 1, 8, 100, 0, 0), (0, 1, 0, 8, 100, 0, 0), (2, 1, 1, 8, 100, 0, 0), (0, 1, 1, 6, 100, 0, 0), (0, 1, 1, 8, 100, -1, 0), (0, 1, 1, 8, 100, 0, -1), (0, 65537, 1, 8, 100, 0, 0),
           (0, 1, 1, 8, 0, 0, 0), (0, 1, 1, 8, 1 << 31, 0, 0)]
    for args in bad:
        assert f(C.byref(c), *args, got) == 1, args
    assert f(C.byref(c), 0, 1, 1, 8, 100, 0, 0, None) == 1 and f(None, 0, 1, 1, 8, 100, 0, 0, got) == 1
    assert f(C.byref(c), 0, 1, (1 << 26) + 1, 8, 100, 0, 0, got) == 2 and f(C.byref(c), 0, 1, 1 << 26, 8, 100, 0, 0, got) == 0
