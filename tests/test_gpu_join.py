"""Joined attention (kvtc_attend_join) against the float64 oracle."""
import numpy as np
import pytest
import torch

import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_gpu_cache import DEV, host, to_dev

pytestmark = pytest.mark.gpu


def check(out, lse, outs, lses, out_dtype):
    """A weight is off by the exponential (2^-21) and its argument (2^-24 of it, as far as 2^7 before it vanishes: 2^-17), sums of p terms by p 2^-24: 2^-15 of the sum of w |out|, twice, and rounded to out_dtype."""
    want, want_lse = sv.join(outs, lses)
    size, _ = sv.join([np.abs(np.nan_to_num(o)) for o in outs], lses)
    got, got_lse = out.float().cpu().numpy(), lse.cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -16 * size + 2.0 ** (-8 if out_dtype == kv.KVTC_BF16 else -22) * np.abs(want) + 1e-37).all()
    gone = np.isneginf(want_lse)
    assert (np.isneginf(got_lse) == gone).all() and (got[gone] == 0).all()
    assert (np.abs(got_lse[~gone] - want_lse[~gone]) <= 2.0 ** -20 + 2.0 ** -22 * np.abs(want_lse[~gone])).all()


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("out_dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("parts,rows,heads,d", [(1, 3, 1, 64), (2, 64, 32, 128), (3, 17, 5, 256), (7, 1, 1, 128), (16, 33, 3, 64), (5, 700, 4, 128)])
def test_joined_parts_are_the_oracles(dtype, out_dtype, parts, rows, heads, d):
    rng = np.random.default_rng(parts + rows)
    outs = [host(rng.standard_normal((rows, heads, d)).astype(np.float32), dtype) for _ in range(parts)]
    lses = [(rng.standard_normal((rows, heads)) * 10).astype(np.float32) for _ in range(parts)]
    for p in range(parts):
        gone = rng.random((rows, heads)) < 0.3
        lses[p][gone] = -np.inf
        outs[p][gone] = np.nan                                       # whatever it holds
    lses[0].flat[0] = 3e4                                            # one that outweighs all others
    outs[0].reshape(-1, d)[0] = 1.5
    t = torch.bfloat16 if out_dtype == kv.KVTC_BF16 else torch.float32
    out, lse = torch.full((rows + 1, heads, d), 5.0, dtype=t, device=DEV), torch.full((rows + 1, heads), 5.0, device=DEV)
    devs, dev_lses = [to_dev(o, dtype) for o in outs], [torch.from_numpy(x).to(DEV) for x in lses]
    kv.kvtc_attend_join(devs, dev_lses, dtype, rows, heads, d, out, out_dtype, lse)
    torch.cuda.synchronize()
    check(out[:rows], lse[:rows], outs, lses, out_dtype)
    assert bool((out[rows] == 5.0).all()) and bool((lse[rows] == 5.0).all())
    again = torch.empty((rows, heads, d), dtype=t, device=DEV)
    kv.kvtc_attend_join(devs, dev_lses, dtype, rows, heads, d, again, out_dtype)      # without log-sums
    torch.cuda.synchronize()
    assert torch.equal(again, out[:rows])
    if dtype == out_dtype:                                           # into the last part's place
        kv.kvtc_attend_join(devs, dev_lses, dtype, rows, heads, d, devs[-1], out_dtype, dev_lses[-1])
        torch.cuda.synchronize()
        assert torch.equal(devs[-1], out[:rows]) and torch.equal(dev_lses[-1], lse[:rows])


def test_the_same_part_twice_and_infinite_values():
    outs, lse = torch.randn((4, 2, 64), device=DEV), torch.randn((4, 2), device=DEV)
    outs[1, 0, 3], outs[2, 1, 5] = float("inf"), float("nan")
    got, got_lse = torch.empty_like(outs), torch.empty_like(lse)
    kv.kvtc_attend_join([outs, outs], [lse, lse], kv.KVTC_F32, 4, 2, 64, got, kv.KVTC_F32, got_lse)
    torch.cuda.synchronize()
    fine = torch.isfinite(outs)
    assert torch.equal(got[fine], outs[fine]) and bool(torch.isinf(got[1, 0, 3])) and bool(torch.isnan(got[2, 1, 5]))
    assert float((got_lse - lse - np.log(2.0)).abs().max()) < 1e-6
