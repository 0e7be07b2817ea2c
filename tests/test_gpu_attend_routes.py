"""Every kernel that kvtc_attend has, by a call that the host's rules send there (asserted), against the CPU oracle."""
import numpy as np
import pytest
import torch

import paper_2511_01815_amd as kv
from test_attend_route import route
from test_gpu_attend import EDGES, Case
from test_gpu_cache import DEV

pytestmark = pytest.mark.gpu

BF16, F32 = kv.KVTC_BF16, kv.KVTC_F32


def check(case, max_tokens, want, only=None):
    """The call, by the route expected of it on a card of 256 compute units, twice."""
    short = -(-max_tokens // case.page) - case.table.shape[1]
    if short > 0:
        case.table = np.pad(case.table, ((0, 0), (0, short)), constant_values=-5)
        case.table_dev = torch.from_numpy(case.table).to(DEV)
    if torch.cuda.get_device_properties(DEV).multi_processor_count == 256:
        got = route(case.cache, case.dtype, len(case.lengths), case.q.shape[1], max_tokens, case.sinks, case.window)
        assert {k: got[k] for k in want} == want, got
    out, lse, status = case.run(max_tokens=max_tokens)
    again = case.run(max_tokens=max_tokens)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse, only=only)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


# several KV heads to a workgroup: rows of neighbouring heads in one cache line, many items, a bound of many tokens
@pytest.mark.parametrize("fmt,dtype,d,heads,group,max_tokens,pieces,next_", [
    ("fp8", F32, 64, 8, 5, 33000, 1, 2), ("fp8", BF16, 64, 8, 8, 33000, 1, 2), ("int4", F32, 128, 8, 5, 33000, 1, 2), ("int4", F32, 64, 10, 3, 33000, 1, 2),
    ("int4", F32, 64, 8, 4, 33000, 1, 4), ("int4", F32, 64, 16, 1, 33000, 1, 4), ("int4", BF16, 64, 10, 8, 33000, 2, 2), ("int4", BF16, 64, 8, 3, 33000, 2, 4),
    ("int4", BF16, 128, 8, 7, 33000, 2, 2)])
def test_several_heads_to_a_workgroup(fmt, dtype, d, heads, group, max_tokens, pieces, next_):
    lengths = (EDGES + [64, 700, 0, 1025, 2000] + EDGES[:14] * 3)[:64]
    case = Case(np.random.default_rng(d + heads + group), fmt, d, heads, group, 16, "tokens", lengths, dtype)
    check(case, max_tokens, dict(rows=0, next=next_, pieces=pieces), only=range(40))


@pytest.mark.parametrize("fmt,dtype,d,heads,group,sinks,window,pieces,next_", [
    ("int4", BF16, 64, 16, 3, 40, 960, 2, 4), ("int4", F32, 64, 16, 2, 70, 1000, 1, 4), ("int4", BF16, 128, 16, 2, 5, 500, 2, 2), ("int4", F32, 128, 16, 1, 33, 961, 1, 2),
    ("fp8", BF16, 64, 16, 4, 9, 1300, 1, 2), ("fp8", F32, 64, 16, 1, 96, 1090, 1, 2), ("int4", BF16, 64, 18, 5, 9, 1100, 2, 2)])
def test_several_heads_to_a_workgroup_with_windows(fmt, dtype, d, heads, group, sinks, window, pieces, next_):
    """Sinks, what is not seen, and a window, in steps and tiles of the waves that a KV head has."""
    rng = np.random.default_rng(d + group + window)
    lengths = [int(n) for n in rng.integers(0, 40, size=256)]
    lengths[::40] = [window + k for k in (-1, 0, 1, sinks, sinks + 40, 700, 1999)]
    case = Case(rng, fmt, d, heads, group, 32, "tokens", lengths, dtype, sinks, window)
    check(case, 4000, dict(rows=0, next=next_, pieces=pieces), only=list(range(0, 256, 40)) + [1, 2, 3, 255])


# two pieces to a step, over the jump from the sinks' pieces (an odd and an even number) to the window's
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,page,order,sinks,window", [(5, 48, "slab", 5, 200), (1, 128, "tokens", 40, 33), (8, 16, "heads", 70, 100), (4, 64, "heads", 0, 257), (3, 32, "tokens", 96, 31)])
def test_two_pieces_to_a_step_with_windows(d, group, page, order, sinks, window):
    lengths = (EDGES + [n + k for n in (64 * 4, 64 * 8) for k in (-33, -32, -1, 0, 1, 31, 32)] + [sinks + window + k for k in (-1, 0, 1, 30, 31, 32, 33, 64, 95)] + [1500] + EDGES)[:62]
    case = Case(np.random.default_rng(d + group + page), "int4", d, 4, group, page, order, lengths, BF16, sinks, window)
    check(case, 1500, dict(rows=0, next=1, pieces=2))


# rows of up to 1024 tokens by a wave each
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("dtype,d,heads,group,page,order,sinks,window", [(BF16, 128, 16, 4, 16, "heads", 0, 0), (F32, 64, 16, 2, 20, "tokens", 0, 0), (BF16, 256, 8, 3, 64, "heads", 0, 0), (BF16, 64, 16, 1, 32, "slab", 40, 800)])
def test_rows_of_a_thousand_tokens_by_single_waves(fmt, dtype, d, heads, group, page, order, sinks, window):
    lengths = [0, 1, 30, 33] * 33
    lengths[::12] = [513, 544, 545, 800, 841, 960, 991, 992, 993, 1023, 1024]
    case = Case(np.random.default_rng(d + group), fmt, d, heads, group, page, order, lengths, dtype, sinks, window)
    check(case, 1024, dict(rows=1, workgroups=len(lengths) * heads), only=list(range(0, 132, 12)) + [1, 2, 3])


@pytest.mark.parametrize("fmt,dtype,d,heads,lengths", [("int4", BF16, 128, 8, [20000]), ("fp8", BF16, 64, 4, [9001, 0, 4097]), ("int4", F32, 64, 2, [0, 24601])])
def test_shares_in_turn(fmt, dtype, d, heads, lengths):
    """Few items of a multiple of eight shares, whose rows share cache lines."""
    case = Case(np.random.default_rng(d + heads), fmt, d, heads, 2, 64, "tokens", lengths, dtype)
    check(case, max(lengths), dict(rows=0, next=1, in_turn=1))
