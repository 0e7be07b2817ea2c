"""By which kernel a kvtc_attend runs, on the CPU: the rules are the host's."""
import ctypes as C

import pytest

import paper_2511_01815_amd as kv

FORMATS = {"bf16": kv.KVTC_CACHE_BF16, "fp8": kv.KVTC_CACHE_FP8, "int4": kv.KVTC_CACHE_INT4}


def cache_of(fmt, heads, d, page, order="tokens", n_pages=32):
    """A valid descriptor over addresses that are never touched."""
    row = kv.kvtc_cache_row_bytes(FORMATS[fmt], d)
    token, head = (row * heads, row) if order == "tokens" else (row, row * page)
    return kv.cache(FORMATS[fmt], n_pages, page, heads, d, 1 << 20, 2 << 20, row * heads * page, head, token, 3 << 20, 4 << 20)


def route(cache, dtype, n_seqs, n_q_heads, max_tokens, sinks=0, window=0):
    got = (C.c_int32 * 5)()
    assert kv.lib().kvtc_host_attend_route(C.byref(cache), dtype, n_seqs, n_q_heads, max_tokens, sinks, window, got) == 0, kv.kvtc_last_error()
    return dict(zip(("rows", "in_turn", "pieces", "next", "workgroups"), got))


@pytest.mark.parametrize("fmt,d", [("int4", 64), ("int4", 128), ("fp8", 64), ("int4", 256), ("fp8", 128), ("bf16", 64)])
@pytest.mark.parametrize("heads,group", [(4, 1), (4, 4), (8, 2), (2, 8)])
def test_the_tiles_of_all_sequences_are_counted_in_32_bits(fmt, d, heads, group):
    """Sequences that share their pages may have more tokens together than there is memory for: what the kernel adds up must fit for every call that is accepted."""
    cache, accepted = cache_of(fmt, heads, d, 64), 0
    for n_seqs, max_tokens in [(65536, 1 << 21), (65536, (1 << 22) - 200), (65535, (1 << 22) - 200), (32768, (1 << 22) - 32), (128, 2 ** 31 - 1), (129, 2 ** 31 - 1), (63, 2 ** 31 - 1), (255, 1 << 30)]:
        fits = n_seqs * -(-max_tokens // 128) < 1 << 31
        assert (kv.kvtc_attend_work_bytes(cache, n_seqs, heads * group, max_tokens) > 0) == fits
        for dtype in (kv.KVTC_BF16, kv.KVTC_F32) if fits else ():
            for sinks, window in ((0, 0), (1 << 20, 1 << 30)):
                r = route(cache, dtype, n_seqs, heads * group, max_tokens, sinks, window)
                tile = 4 // r["next"] * r["pieces"]
                assert r["rows"] or -(-(-(-max_tokens // 32)) // tile) * n_seqs < 1 << 32, (n_seqs, max_tokens, r)
                accepted += 1
    assert accepted >= 20


def test_refusals_of_the_route():
    c = cache_of("fp8", 4, 64, 16)
    f, got = kv.lib().kvtc_host_attend_route, (C.c_int32 * 5)()
    assert f(C.byref(c), 2, 1, 8, 100, 0, 0, got) == 1 and f(C.byref(c), 0, 1, 6, 100, 0, 0, got) == 1 and f(C.byref(c), 0, 1, 8, 100, -1, 0, got) == 1 and f(C.byref(c), 0, 1, 8, 100, 0, 0, None) == 1
    assert f(C.byref(c), 0, 65536, 8, 1 << 23, 0, 0, got) == 2 and f(None, 0, 1, 8, 100, 0, 0, got) == 1


def test_several_heads_to_a_workgroup_take_two_pieces_where_any_do():
    """Of 4 bits with bf16 queries there is no kernel of several heads and one piece to a step; the others have one piece only."""
    seen = set()
    for fmt, dtype in (("int4", kv.KVTC_BF16), ("int4", kv.KVTC_F32), ("fp8", kv.KVTC_BF16)):
        for d in (64, 128):
            for heads, group in ((2, 1), (2, 8), (4, 3), (8, 2), (16, 1), (64, 5), (1024, 1)):
                for n_seqs in (1, 3, 24, 48, 256, 4096, 65536):
                    for max_tokens in (1, 33, 700, 2048, 4097, 16384, 33000):
                        for sinks, window in ((0, 0), (4, 128), (1000, 3000)):
                            r = route(cache_of(fmt, heads, d, 16), dtype, n_seqs, heads * group, max_tokens, sinks, window)
                            assert r["next"] == 1 or not r["rows"] and r["pieces"] == (2 if (fmt, dtype) == ("int4", kv.KVTC_BF16) else 1), (fmt, dtype, d, heads, group, n_seqs, max_tokens, r)
                            seen.add((fmt, dtype, d, r["next"], r["pieces"]))
    assert {(f, t, d, n) for f, t, d, n, _ in seen if n > 1} == {("int4", t, d, n) for t in (kv.KVTC_BF16, kv.KVTC_F32) for d, n in ((64, 2), (64, 4), (128, 2))} | {("fp8", kv.KVTC_BF16, 64, 2)}


def test_shares_in_turn_only_where_the_same_tokens_fall_to_one_xcd():
    """In turn, share i is XCD i % 8's: the shares of different heads that read the same tokens meet there where every item has a multiple of eight."""
    seen = set()
    for fmt, d, dtype in (("int4", 128, kv.KVTC_BF16), ("int4", 64, kv.KVTC_F32), ("fp8", 64, kv.KVTC_BF16)):
        for heads in (1, 2, 3, 4, 5, 7, 8, 10, 12, 16, 24):
            for n_seqs in (1, 2, 3, 5, 16):
                for max_tokens in (700, 4096, 131072):
                    r = route(cache_of(fmt, heads, d, 64), dtype, n_seqs, heads * 4, max_tokens)
                    even = r["workgroups"] % (8 * heads * n_seqs) == 0
                    assert not r["in_turn"] or even and r["next"] == 1 and heads * n_seqs <= 16, (fmt, d, heads, n_seqs, max_tokens, r)
                    seen.add((r["in_turn"], even))
                    assert not route(cache_of(fmt, heads, d, 64, "heads"), dtype, n_seqs, heads * 4, max_tokens)["in_turn"] or heads == 1
    assert (1, True) in seen
