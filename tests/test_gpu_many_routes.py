"""Every kernel of kvtc_attend_many, whole and in parts, at sizes by which its rule picks it."""
import numpy as np
import pytest
import torch

import paper_2511_01815_amd as kv
from test_attend_route import cache_of
from test_gpu_cache import FORMATS
from test_gpu_many import Case
from test_many_route import route

pytestmark = pytest.mark.gpu

# (heads, group, new tokens, tokens before)
CALLS = [(1, 1, [1], [0]), (2, 3, [1], [699]), (2, 1, [1, 1], [699, 20]), (1, 1, [1], [199]), (1, 1, [1], [1999]), (2, 1, [1] * 64, [i % 5 for i in range(64)]), (32, 6, [2] * 40 + [60], [i % 4 for i in range(41)]),
         (8, 4, [33], [3967]), (4, 4, [9, 7], [7991, 300]), (32, 4, [150], [0]), (32, 6, [150], [0]), (32, 1, [1], [7999]), (1, 1, [1] * 5, [3999, 0, 64, 31, 700]), (1, 1, [17, 0] + [16] * 14, [7983] + [100] * 15),
         (2, 1, [1] * 64, [7999] + [33] * 63), (1, 1, [300] + [200] * 15, [3700] + [i for i in range(15)]), (4, 4, [33, 31], [7967, 700]),
         (32, 6, [33] * 64, [0] * 64), (1, 1, [300] * 16, [3700] + [9 * i for i in range(15)]), (4, 4, [7, 7], [7993, 300]), (4, 6, [33] * 64, [0] * 64), (8, 4, [33] * 64, [0] * 64),
         (32, 1, [1], [11999]), (4, 1, [1], [8999]), (1, 1, [1] * 16, [3999] + [7 * i for i in range(15)])]


def reached(fmt, d):
    """{(kernel, in parts): the call that takes least}, of bf16 queries."""
    found = {}
    for heads, group, new, had in CALLS:
        most = max(n + h for n, h in zip(new, had))
        r = route(cache_of(fmt, heads, d, 16), kv.KVTC_BF16, len(new), sum(new) + 2, heads * group, most)
        work = sum(n * (n + h) for n, h in zip(new, had)) * heads * group
        if (r["kind"], r["parts"] > 1) not in found or work < found[r["kind"], r["parts"] > 1][0]:
            found[r["kind"], r["parts"] > 1] = (work, heads, group, new, had, r["parts"])
    return found


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,parts", [(k, p) for k in (1, 2, 3) for p in (False, True)])
def test_kernels_whole_and_in_parts(fmt, d, kind, parts):
    found = reached(fmt, d)
    if (kind, parts) not in found:
        assert (kind, parts) == (2, True) and fmt != "bf16" and d < 256, (kind, parts, sorted(found))     # (the rule does not take it at such sizes)
        return
    _, heads, group, new, had, n = found[kind, parts]
    case = Case(np.random.default_rng(kind + 3 * n + d), fmt, d, heads, group, 16, "heads", new, had, kv.KVTC_BF16)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse, only=sorted({0, 1, len(new) - 1} & set(range(len(new)))))


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_as_many_sequences_as_a_call_takes(dtype):
    """65536 sequences of one new token: more items than 16 bits count."""
    case = Case(np.random.default_rng(5), "fp8", 64, 1, 2, 16, "tokens", [1] * 65536, [i % 7 for i in range(65536)], dtype)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse, only={0, 1, 6, 77, 32767, 32768, 65534, 65535})
