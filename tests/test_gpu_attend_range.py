"""kvtc_attend where single roundings and the ends of number ranges show: rows made by hand, whose exact result and whose rounding errors are worked out here in
float64."""
import numpy as np
import pytest
import torch

import kvtc_paged as kp
import paper_2511_01815_amd as kv
from test_gpu_attend import Work
from test_gpu_cache import DEV, Pool, host, to_dev

pytestmark = pytest.mark.gpu


class Rows:
    """One sequence and KV head; keys and values of every token by hand."""

    def __init__(self, fmt, d, n, q, dtype, scale=1.0, page=64):
        self.fmt, self.d, self.n, self.dtype, self.scale = fmt, d, n, dtype, scale
        self.pool = Pool(fmt, -(-n // page), page, 1, d)
        self.q = host(np.atleast_2d(np.asarray(q, np.float32)), dtype)

    def codes(self, side, token, codes, scale, shift=0.0):
        """A token's row: 8 bits, codes as values and one scale; 4 bits, one code, scale and shift for all features."""
        r, s = self.pool.at(token, 0)
        if self.fmt == "fp8":
            self.pool.bytes[side][r:r + self.d] = kp.e4m3_codes(np.broadcast_to(codes, self.d))
            self.pool.scales[side][s:s + 4] = np.array([scale], np.float32).view(np.uint8)
        else:
            self.pool.bytes[side][r:r + self.d // 2] = codes * 17
            self.pool.scales[side][s:s + self.pool.scale] = np.tile(np.array([shift, scale], np.float16), self.d // 32).view(np.uint8)

    def values(self, side, token, x):
        """A token's row of bf16 features."""
        r, _ = self.pool.at(token, 0)
        self.pool.bytes[side][r:r + 2 * self.d] = kp.bf16_bits(np.broadcast_to(np.asarray(x, np.float32), self.d)).view(np.uint8)

    def held(self, side):
        rows, scales = self.pool.rows(side, range(self.n), 0)
        return kp.values(rows, scales, self.fmt, self.d)

    def run(self):
        cache, hq = self.pool.upload(), self.q.shape[0]
        q = to_dev(self.q, self.dtype)[None].contiguous()
        pages = torch.arange(self.pool.n_pages, dtype=torch.int32, device=DEV)[None]
        work = Work.get(kv.kvtc_attend_work_bytes(cache, 1, hq, self.n))
        out, lse = torch.full_like(q, 5.0), torch.full((1, hq), 5.0, device=DEV)
        kv.kvtc_attend(cache, q, self.dtype, 1, hq, hq * self.d, self.d, pages, pages.shape[1], torch.tensor([self.n], dtype=torch.int32, device=DEV), self.n, self.scale,
                       0, 0, out, lse, work, work.numel())
        torch.cuda.synchronize()
        return out[0].float().cpu().numpy().astype(np.float64), lse[0].cpu().numpy().astype(np.float64)


def cut_error(p):
    """What is lost of p by two parts of 8 bits, the first towards zero, the second to nearest."""
    first = (p.astype(np.float32).view(np.uint32) & 0xFFFF0000).view(np.float32).astype(np.float64)
    rest = p - first
    return rest - kp.bf16_value(kp.bf16_bits(rest.astype(np.float32))).astype(np.float64)


@pytest.mark.parametrize("fmt", ["fp8", "int4"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_probabilities_of_codes_have_18_bits(fmt, d):
    """Values that cancel, with probabilities that two parts cut towards zero would miss by nearly 2^-16 each, in one direction.  A probability is off by 2^-18 (two parts to nearest) and 2^-21 (the
    exponential, the score), sums of n tokens by (n + 4) 2^-24 of their magnitudes (4 bits: whole bytes are 17 codes, of which a 16th counts), the result by bf16's rounding."""
    x = np.arange(0.55, 0.69, 2.0 ** -11).astype(np.float16).astype(np.float64)
    p = np.exp(-x)
    err = cut_error(p)
    down = np.argsort(-err)[:3]                                  # too small by the most
    n = 7
    q = np.zeros(d)
    q[0] = 1.0
    rows = Rows(fmt, d, n, q, kv.KVTC_BF16)
    weight = np.ones(n)
    if fmt == "int4":
        assert (err[down] > 0.8 * 2.0 ** -17).all()
        for t in range(n):
            i = down[(t - 1) // 2]
            rows.codes(0, t, 0, 0.0, 0.0 if t == 0 else -x[i])
            rows.codes(1, t, *((0, 0.0) if t == 0 else (15, 1.0) if t % 2 else (0, 0.0, -15.0)))
            weight[t] = 1.0 if t == 0 else p[i]
        size = 17.0 * weight[1::2].sum(), 32.0 * weight[1::2].sum()
    else:
        fine = x[down][:, None] + np.arange(-400, 400) * 2.0 ** -20      # near each, one too small by about as much and one too large
        e = cut_error(np.exp(-fine))
        pairs = [(fine[k, e[k].argmax()], fine[k, e[k].argmin()]) for k in range(3)]
        for t in range(n):
            if t:
                at = pairs[(t - 1) // 2][(t - 1) % 2]
                weight[t] = np.exp(-np.float64(np.float32(at)))
            rows.codes(0, t, -1.0 if t else 0.0, np.float32(at) if t else 1.0)
            rows.codes(1, t, 0.0 if t == 0 else 1.0 if t % 2 else -1.0, 1.0)
        assert (e.max(1) > 0.8 * 2.0 ** -17).all() and (e.min(1) < -0.8 * 2.0 ** -17).all()
        size = weight[1:].sum(), weight[1:].sum()
    want, want_lse = kp.attend(rows.q, rows.held(0), rows.held(1), 1.0)
    np.testing.assert_allclose(want_lse, np.log(weight.sum()), rtol=1e-6)
    out, lse = rows.run()
    tol = ((2.0 ** -18 + 2.0 ** -21) * size[0] + (n + 4) * 2.0 ** -24 * size[1]) / weight.sum() + 2.0 ** -9 * np.abs(want)
    assert (np.abs(out - want) <= tol).all(), (np.abs(out - want).max(), tol.min())
