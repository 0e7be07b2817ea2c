"""kvtc_attend_many over 8 and 4 bits: rows whose largest probability falls to a token without values, so that all of the result is of tokens far below it."""
import numpy as np
import pytest
import torch

import kvtc_paged as kp
import paper_2511_01815_amd as kv
from test_gpu_many import Case, bits_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("below", [10, 19, 25])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("fmt", ["fp8", "int4"])
@pytest.mark.parametrize("new,had", [([6], [1500]), ([200, 3], [10, 300])])
def test_all_of_the_result_below_the_largest(fmt, d, new, had, below):
    """Probabilities are fp16 numbers, 2^6 times what they are of the largest so far: 11 bits (off by 2^-11 of themselves) down to 2^-20 of it, and off by 2^-31 of it below.  Over 8 bits they are times their values'
    scales, of the largest so far, and the error is times a code: 2^-31 of the largest value again."""
    rng = np.random.default_rng(below + d)
    case = Case(rng, fmt, d, 1, 4, 16, "heads", new, had, kv.KVTC_BF16)
    case.q[..., 0] = 8.0
    case.q_dev[..., 0] = 8.0
    score = (below + 4) * np.log(2.0)                                # (the others' scores are of 0 +- 2.5 or so)
    for b, n in enumerate(case.lengths):
        x = [rng.standard_normal((n, 1, d)).astype(np.float32) for _ in range(2)]
        x[0][..., 0] = 0.0
        x[0][0], x[1][0] = 0.0, 0.0
        x[0][0, :, 0] = score / (case.scale * 8.0)
        for side in range(2):
            case.pool.put(side, case.slots[b], x[side])
    case.upload()
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    _, kept, value, result = bits_of(fmt, kv.KVTC_BF16)
    weights = []
    for b, n in enumerate(case.new):
        k, v = [kp.values(*case.pool.rows(side, case.slots[b], 0), fmt, d) for side in range(2)]
        for i in range(n):
            r, t = case.starts[b] + i, case.lengths[b] - n + i + 1
            if t < 2:
                continue
            want, want_lse = kp.attend(case.q[r], k[:t], v[:t], case.scale)
            size = np.abs(k[:t]) if fmt == "fp8" else 3 * np.repeat(np.abs(k[:t]).reshape(t, -1, 32).max(-1), 32, axis=1)
            tol, tol_lse = kp.attend_bound(case.q[r], k[:t], v[:t], size, np.abs(v[:t]), case.scale, kept, result)
            p = np.exp(case.scale * (case.q[r] @ k[:t].T) - want_lse[:, None])
            tol = tol + 2.0 ** -value * (p @ np.abs(v[:t])) + t * 2.0 ** -31 * np.abs(v[:t]).max()
            assert (np.abs(out[r] - want) <= tol).all(), (b, i, np.abs(out[r] - want).max(), tol.min())
            assert (np.abs(lse[r] - want_lse) <= tol_lse).all()
            weights.append(np.median(p[:, 1:]))
    assert 2.0 ** (-below - 8) < np.median(weights) < 2.0 ** -below   # (what the test is about)
