"""kvtc_attend where its kernels change: many short rows (a wave to each), 4-bit rows of which a step takes two pieces, rows joined from hundreds of parts, and large
writes and reads (several rows to a lane), each against the CPU oracle."""
import numpy as np
import pytest
import torch

import kvtc_paged as kp
import paper_2511_01815_amd as kv
from test_gpu_attend import EDGES, Case
from test_gpu_cache import DEV, FORMATS, Pool, features, host, to_dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype,d,group,page,order,sinks,window", [(kv.KVTC_BF16, 128, 4, 16, "heads", 0, 0), (kv.KVTC_BF16, 64, 3, 7, "tokens", 0, 0), (kv.KVTC_F32, 128, 1, 32, "tokens", 3, 50),
                                                                  (kv.KVTC_BF16, 256, 5, 64, "slab", 0, 0), (kv.KVTC_F32, 64, 17, 48, "heads", 0, 9)])
def test_many_short_rows(fmt, dtype, d, group, page, order, sinks, window):
    """2048 items and more, rows of at most 16 pieces of 32 tokens; invalid lengths among them."""
    rng = np.random.default_rng(d + group)
    lengths = (EDGES[:18] * 15)[:258]
    case = Case(rng, fmt, d, 8, group, page, order, lengths, dtype, sinks, window)
    bad = list(lengths)
    bad[200], bad[31] = -1, 513
    case.lengths_dev = torch.tensor(bad, dtype=torch.int32, device=DEV)
    case.slots[200] = case.slots[31] = np.zeros(0, np.int64)
    case.table = np.pad(case.table, ((0, 0), (0, 512)), constant_values=-7)      # (a table for 512 tokens and more)
    case.table_dev = torch.from_numpy(case.table).to(DEV)
    out, lse, status = case.run(max_tokens=512)
    torch.cuda.synchronize()
    assert int(status.item()) == 32
    case.check(out, lse, only=list(range(0, 258, 5)) + [31, 200, 257])
    assert bool(torch.isfinite(out.float()).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,page,order,sinks,window", [(4, 16, "heads", 0, 0), (8, 64, "tokens", 0, 0), (5, 48, "slab", 5, 200), (1, 128, "tokens", 40, 33), (9, 16, "heads", 0, 0)])
def test_four_bits_at_every_edge_of_a_step(d, group, page, order, sinks, window):
    """Enough to do for two pieces to a step, where the query heads fit half of the columns (9 do not); lengths around every piece, step and tile, the largest of many tiles."""
    lengths = EDGES + [n + k for n in (64 * 4, 64 * 8, 64 * 16) for k in (-33, -32, -1, 0, 1, 31, 32)] + [3001]
    case = Case(np.random.default_rng(d + group + page), "int4", d, 2, group, page, order, lengths, kv.KVTC_BF16, sinks, window)
    out, lse, status = case.run(max_tokens=3001)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse)


@pytest.mark.parametrize("fmt,dtype,d,group,tokens", [("fp8", kv.KVTC_BF16, 128, 16, 40000), ("bf16", kv.KVTC_BF16, 64, 1, 66000), ("int4", kv.KVTC_F32, 256, 3, 33000), ("int4", kv.KVTC_BF16, 128, 2, 70000)])
def test_rows_of_hundreds_of_parts(fmt, dtype, d, group, tokens):
    case = Case(np.random.default_rng(tokens), fmt, d, 1, group, 64, "heads", [tokens], dtype)
    first = case.run()
    again = case.run()
    torch.cuda.synchronize()
    case.check(first[0], first[1])
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_fewer_tiles_than_shares():
    """A bound of many tokens, rows of few: fewer tiles in all than the launch has workgroups, so that some have nothing to do, and none is waited for."""
    for fmt in FORMATS:
        case = Case(np.random.default_rng(1), fmt, 128, 2, 4, 64, "heads", [130, 0, 400, 1], kv.KVTC_BF16)
        case.table = np.pad(case.table, ((0, 0), (0, 2000)))
        case.table_dev = torch.from_numpy(case.table).to(DEV)
        for _ in range(3):
            out, lse, status = case.run(max_tokens=100_000)
            torch.cuda.synchronize()
            assert int(status.item()) == 0
            case.check(out, lse)


@pytest.mark.parametrize("fmt", ["fp8", "int4"])
@pytest.mark.parametrize("d,heads,n,page,order", [(128, 8, 16411, 64, "heads"), (64, 5, 52501, 20, "tokens"), (256, 2, 32793, 128, "slab")])
def test_large_calls_are_small_ones_side_by_side(fmt, d, heads, n, page, order):
    """From two million lanes on a lane has several rows: the same bytes and values as calls of a few thousand tokens, which the oracle checks elsewhere; some rows by the oracle here."""
    rng = np.random.default_rng(n)
    n_pages = -(-n // page) + 1
    slots = torch.from_numpy(rng.permutation(n_pages * page)[:n].astype(np.int64)).to(DEV)
    slots[5] = -1
    slots[n - 2] = n_pages * page
    gen = torch.Generator(device=DEV).manual_seed(n)
    x = [(torch.randn((n, heads, d), generator=gen, device=DEV) * 3).to(torch.bfloat16) for _ in range(2)]
    x[0][:7] = to_dev(features(rng, (7, heads, d)), kv.KVTC_BF16)
    pools = [Pool(fmt, n_pages, page, heads, d, order) for _ in range(2)]
    caches = [p.upload() for p in pools]
    status = torch.zeros(2, dtype=torch.int32, device=DEV)
    outs = [[torch.full_like(x[0], 3.0) for _ in range(2)] for _ in range(2)]
    kv.kvtc_cache_write(caches[0], x[0], x[1], kv.KVTC_BF16, n, heads * d, d, slots, status[0:1])
    kv.kvtc_cache_read(caches[0], slots, n, outs[0][0], outs[0][1], kv.KVTC_BF16, heads * d, d, status[1:2])
    for at in range(0, n, 3000):
        m = min(3000, n - at)
        kv.kvtc_cache_write(caches[1], x[0][at:], x[1][at:], kv.KVTC_BF16, m, heads * d, d, slots[at:])
        kv.kvtc_cache_read(caches[1], slots[at:], m, outs[1][0][at:], outs[1][1][at:], kv.KVTC_BF16, heads * d, d)
    torch.cuda.synchronize()
    assert status.cpu().tolist() == [n - 1, n - 1]
    for side in range(2):
        assert torch.equal(pools[0].dev[side], pools[1].dev[side]) and torch.equal(pools[0].dev_scales[side], pools[1].dev_scales[side])
        assert torch.equal(outs[0][side], outs[1][side])
        some = list(range(0, 5)) + [6, 999, n // 2, n - 1]
        rows, scales = kp.quantise(x[side][some].float().cpu().numpy(), fmt)
        want = host(kp.values(rows, scales, fmt, d).astype(np.float32), kv.KVTC_BF16)
        np.testing.assert_array_equal(outs[0][side][some].float().cpu().numpy(), want)
        assert bool((outs[0][side][5] == 0).all()) and bool((outs[0][side][n - 2] == 0).all())


@pytest.mark.parametrize("fmt,dtype,d,heads,group,sinks,window", [("int4", kv.KVTC_BF16, 128, 8, 4, 0, 0), ("int4", kv.KVTC_BF16, 64, 8, 4, 0, 0), ("int4", kv.KVTC_BF16, 64, 6, 7, 9, 700), ("fp8", kv.KVTC_BF16, 64, 8, 5, 0, 0),
                                                                  ("fp8", kv.KVTC_F32, 64, 4, 8, 0, 0), ("fp8", kv.KVTC_BF16, 64, 8, 16, 0, 0)])
def test_token_major_heads_that_share_a_cache_line(fmt, dtype, d, heads, group, sinks, window):
    """Rows of 32 and 64 bytes side by side, and a bound of tokens that makes the call a large one: several KV heads to a workgroup (as far as 16 columns hold their query heads)."""
    lengths = EDGES + [64, 700, 0, 1025, 2000] * 5
    case = Case(np.random.default_rng(d + heads + group), fmt, d, heads, group, 16, "tokens", lengths, dtype, sinks, window)
    case.table = np.pad(case.table, ((0, 0), (0, 2100)))
    case.table_dev = torch.from_numpy(case.table).to(DEV)
    out, lse, status = case.run(max_tokens=33000)
    again = case.run(max_tokens=33000)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d,group", [(64, 4), (128, 4), (128, 16), (256, 3)])
@pytest.mark.parametrize("up,size", [(-60, 0), (50, 0), (100, 0), (0, -16), (-40, 10), (20, -12)])
def test_four_bits_of_any_magnitude(dtype, d, group, up, size):
    """Queries of 2^up and keys and values of 2^size (fp16 headers below the normal numbers among them), the scale such that scores are as ever; a query of zeros, and a feature far above the rest."""
    rng = np.random.default_rng(d + group + up)
    case = Case(rng, "int4", d, 2, group, 32, "heads", [1, 33, 700, 2100], dtype)
    for b, slots in enumerate(case.slots):
        for side in range(2):
            case.pool.put(side, slots, (rng.standard_normal((len(slots), 2, d)) * 2.0 ** size).astype(np.float32))
    case.cache = case.pool.upload()
    case.q[0, 0] = 0
    case.q[2, :, 5] *= 64
    case.q = host((case.q * 2.0 ** up).astype(np.float32), dtype)
    case.q_dev = to_dev(case.q, dtype)
    case.scale = d ** -0.5 * 2.0 ** -(up + size)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and bool(torch.isfinite(lse).all())
    case.check(out, lse)


@pytest.mark.parametrize("fmt,d,heads", [("int4", 128, 4), ("int4", 64, 4), ("fp8", 64, 3)])
def test_few_long_token_major_rows(fmt, d, heads):
    """Few items whose rows share cache lines: shares go to the XCDs in turn."""
    case = Case(np.random.default_rng(d + heads), fmt, d, heads, 2, 64, "tokens", [9001, 0, 4097], kv.KVTC_BF16)
    first, again = case.run(), case.run()
    torch.cuda.synchronize()
    case.check(first[0], first[1])
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
