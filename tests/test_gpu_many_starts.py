"""Starts that do not ascend or leave the batch: kvtc_attend_many leaves those sequences' rows as they are, and works out all others'."""
import numpy as np
import pytest
import torch

import kvtc_paged as kp
import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_gpu_many import Case, DEV, bits_of

pytestmark = pytest.mark.gpu


def run(case, starts, most):
    """The call with these starts, against float64; which rows have to stay."""
    served, bad = sv.served(starts, case.rows)
    case.starts_dev = torch.from_numpy(np.asarray(starts, np.int32)).to(DEV)
    out, lse, status = case.run(max_tokens=most)
    torch.cuda.synchronize()
    assert int(status.item()) == bad
    out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    untouched = np.ones(case.rows, bool)
    for b in served:
        s0, n = starts[b], starts[b + 1] - starts[b]
        assert untouched[s0:s0 + n].all()
        untouched[s0:s0 + n] = False
        if len(served) > 600 and b % 8:
            assert (lse[s0:s0 + n] != 5.0).all()
            continue
        for h in range(case.heads):
            k, v = [kp.values(*case.pool.rows(side, case.slots[b], h), case.fmt, case.d) for side in range(2)]
            at = slice(h * case.group, (h + 1) * case.group)
            for i in range(n):
                t = sv.seen(case.lengths[b] - n + i, case.lengths[b], True, 0, 0)
                want, want_lse = kp.attend(case.q[s0 + i, at], k[t], v[t], case.scale)
                tol, tol_lse = sv.bound(case.q[s0 + i, at], k[t], v[t], case.scale, *bits_of(case.fmt, case.dtype))
                assert (np.abs(out[s0 + i, at] - want) <= tol).all(), (b, h, i)
                assert np.isneginf(lse[s0 + i, at]).all() if len(t) == 0 else (np.abs(lse[s0 + i, at] - want_lse) <= tol_lse).all(), (b, h, i)
    assert (out[untouched] == 5.0).all() and (lse[untouched] == 5.0).all()


# What is wrong with a batch's starts: {which: what it becomes}
SPOILT = [{2: -1000000}, {2: 3}, {3: 5, 4: 2}, {1: 1 << 30}, {0: -1}, {3: 100, 5: 0}, {0: 40}, {6: 0}, {6: 1 << 30}, {1: -2 ** 31, 4: 2 ** 31 - 1}, {k: 120 - 20 * k for k in range(7)}]


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("fmt,group", [("bf16", 4), ("fp8", 1)])
@pytest.mark.parametrize("spoilt", SPOILT, ids=str)
def test_a_few_sequences(dtype, fmt, group, spoilt):
    case = Case(np.random.default_rng(len(spoilt) + group), fmt, 64, 1, group, 16, "heads", [40, 1, 33, 2, 60, 7], [30, 200, 0, 64, 5, 100], dtype)
    starts = case.starts.copy()
    for k, v in spoilt.items():
        starts[k] = v
    run(case, starts, max(case.lengths))


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_sequences_in_parts(dtype):
    """What one is left out of does not change how others' parts are joined."""
    case = Case(np.random.default_rng(3), "bf16", 64, 1, 4, 16, "heads", [6, 3, 1, 2], [9001, 300, 4000, 0], dtype)
    for spoilt in ({2: -7}, {1: 1 << 30}, {2: 2}):
        starts = case.starts.copy()
        for k, v in spoilt.items():
            starts[k] = v
        run(case, starts, 9007)


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("n_seqs", [63, 64, 65, 128, 255, 256, 257, 511, 512, 513, 1024, 1025, 3333])
def test_many_sequences(dtype, n_seqs):
    """As few as a wave looks at, and as many as a launch of its own does."""
    rng = np.random.default_rng(n_seqs)
    new, had = rng.integers(0, 4, n_seqs), rng.integers(0, 40, n_seqs)
    new[rng.integers(0, n_seqs, 2)] = 70
    had[new == 0] = 0                                                # (rows that the starts give them see no token)
    case = Case(rng, "fp8", 64, 1, 2, 16, "heads", [int(n) for n in new], [int(n) for n in had], dtype)
    most = max(case.lengths)
    run(case, case.starts.copy(), most)
    for _ in range(3):
        starts = case.starts.copy()
        for k in rng.integers(0, n_seqs + 1, 1 + n_seqs // 200):
            starts[k] += rng.choice([-2 ** 30, -50, -1, 50, 2 ** 30])
        run(case, starts, most)
