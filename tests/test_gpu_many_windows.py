"""kvtc_attend_many with bf16 queries by every kernel, whole and in parts: with sinks and windows, over pages of 16 tokens and of 20, over tokens of another length.  Where no key is rounded, lse is held to what fp32
sums of exact products give."""
import functools

import numpy as np
import pytest
import torch

import kvtc_paged as kp
import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_attend_route import cache_of
from test_gpu_cache import FORMATS
from test_gpu_many import Case, bits_of
from test_gpu_many_routes import reached
from test_many_route import route

pytestmark = pytest.mark.gpu

GROUPS = [(1, 4), (2, 3), (4, 4), (4, 5), (8, 4), (1, 1)]
TOKENS = [([6], [3000]), ([6], [9000]), ([33], [5000]), ([100], [3000]), ([1000], [500]), ([9, 7], [3991, 300]), ([1] * 4, [5000, 100, 3000, 7]), ([40, 33], [4000, 2000])]
WINDOWS = [(4, 2500), (4, 1000), (70, 600), (300, 3000)]


@functools.lru_cache(None)
def windowed(fmt, d):
    """{(kernel, in parts): the calls that take least, one to a window}."""
    found = {}
    for heads, group in GROUPS:
        for new, had in TOKENS:
            for sinks, window in WINDOWS:
                r = route(cache_of(fmt, heads, d, 16), kv.KVTC_BF16, len(new), sum(new) + 2, heads * group, max(n + h for n, h in zip(new, had)), sinks, window)
                work = sum(n * min(n + h, sinks + window) for n, h in zip(new, had)) * heads * group
                mine = found.setdefault((r["kind"], r["parts"] > 1), {})
                if (sinks, window) not in mine or work < mine[sinks, window][0]:
                    mine[sinks, window] = (work, heads, group, new, had, sinks, window)
    return {k: sorted(v.values(), key=lambda c: c[0]) for k, v in found.items()}


def some_rows(new):
    """Of each sequence: all where they are few, else the first, the last and some between them."""
    n = max(new)
    return None if n <= 40 else sorted({0, n - 1} | set(range(3, n, 61)))


def check(case, out, lse, only=None):
    """Case.check() at some rows (and of some sequences), with bounds in which keys enter exactly.  lse: fp32 sums of products of codes (or bf16 numbers) and queries, times scales; over 4 bits of codes times a group's scale and of its shift,
    whose magnitudes are at most 3 times the group's largest value (its least and largest have the codes 0 and 15)."""
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    _, kept, value, result = bits_of(case.fmt, case.dtype)
    for b, n in enumerate(case.new):
        if only is not None and b not in only:
            continue
        for h in range(case.heads):
            k, v = [kp.values(*case.pool.rows(side, case.slots[b], h), case.fmt, case.d) for side in range(2)]
            at = slice(h * case.group, (h + 1) * case.group)
            for i in range(n) if some_rows(case.new) is None else [i for i in some_rows(case.new) if i < n]:
                t = sv.seen(case.lengths[b] - n + i, case.lengths[b], case.causal, case.sinks, case.window)
                q, r = case.q[case.starts[b] + i, at], case.starts[b] + i
                size = np.abs(k[t]) if case.fmt != "int4" else 3 * np.repeat(np.abs(k[t]).reshape(len(t), -1, 32).max(-1), 32, axis=1)
                want, want_lse = kp.attend(q, k[t], v[t], case.scale)
                tol, tol_lse = kp.attend_bound(q, k[t], v[t], size, np.abs(v[t]), case.scale, kept, result)
                tol = tol + 2.0 ** -value * (np.exp(case.scale * (q @ k[t].T) - want_lse[:, None]) @ np.abs(v[t]))
                assert (np.abs(out[r, at] - want) <= tol).all(), (b, h, i, np.abs(out[r, at] - want).max(), tol.min())
                assert (np.abs(lse[r, at] - want_lse) <= tol_lse).all(), (b, h, i, np.abs(lse[r, at] - want_lse).max(), tol_lse.min())


@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,parts", [(k, p) for k in (1, 2, 3) for p in (False, True)])
def test_windows_by_every_kernel(fmt, d, kind, parts, page):
    calls = windowed(fmt, d).get((kind, parts))
    if not calls:
        pytest.skip("the rule takes this kernel so at none of these sizes")
    for _, heads, group, new, had, sinks, window in calls[:3]:
        case = Case(np.random.default_rng(d + kind + page), fmt, d, heads, group, page, "heads", new, had, kv.KVTC_BF16, True, sinks, window)
        out, lse, status = case.run()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        check(case, out, lse)


@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,parts", [(k, p) for k in (1, 2, 3) for p in (False, True)])
def test_tokens_of_another_length_by_every_kernel(fmt, d, kind, parts, page):
    found = reached(fmt, d).get((kind, parts))
    if not found:
        pytest.skip("the rule takes this kernel so at none of these sizes")
    _, heads, group, new, had, _ = found
    case = Case(np.random.default_rng(d + kind + page), fmt, d, heads, group, page, "tokens", new, [n + h for n, h in zip(new, had)], kv.KVTC_BF16, causal=False)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    check(case, out, lse, {0, 1, len(new) - 1})


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,had", [([1, 2, 5], [0, 3, 0]), ([33, 1, 64], [0, 700, 200]), ([130], [1500])])
def test_sums_are_those_of_the_caches_own_keys(fmt, d, new, had):
    """As test_sums_over_four_bits_are_those_of_the_caches_own_keys: no key is rounded over 16 and 8 bits either (a key in 11 bits would be off by 2^-12 of every product on average)."""
    case = Case(np.random.default_rng(d + len(new)), fmt, d, 2, 3, 16, "heads", new, had, kv.KVTC_BF16)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    check(case, out, lse)
