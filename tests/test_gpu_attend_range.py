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


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_probabilities_keep_their_bits(fmt, d):
    """Values that cancel, with probabilities that two parts cut towards zero would miss by nearly 2^-16 each, in one direction.  A probability is off by nothing (three parts) or 2^-18 (4 bits: two parts
    to nearest) and 2^-21 (the exponential, the score), sums of n tokens by (n + 4) 2^-24 of their magnitudes (4 bits: whole bytes are 17 codes, of which a 16th counts), the result by bf16's rounding."""
    x = np.arange(0.55, 0.69, 2.0 ** -11).astype(np.float16).astype(np.float64)
    p = np.exp(-x)
    err = cut_error(p)
    down = np.argsort(-err)[:3]                                  # too small by the most
    n = 7
    q = np.zeros(d)
    q[:3] = 1.0, 2.0 ** -8, 2.0 ** -16
    rows = Rows(fmt, d, n, q if fmt == "bf16" else q * (q == 1.0), kv.KVTC_BF16)
    weight = np.ones(n)
    if fmt == "int4":
        assert (err[down] > 0.8 * 2.0 ** -17).all()
        for t in range(n):
            i = down[(t - 1) // 2]
            rows.codes(0, t, 0, 0.0, 0.0 if t == 0 else -x[i])
            rows.codes(1, t, *((0, 0.0) if t == 0 else (15, 1.0) if t % 2 else (0, 0.0, -15.0)))
            weight[t] = 1.0 if t == 0 else p[i]
        off = 2.0 ** -18 * 17.0 * weight[1::2].sum()
        size = 32.0 * weight[1::2].sum()
    else:
        fine = x[down][:, None] + np.arange(-400, 400) * 2.0 ** -20      # near each, one too small by about as much and one too large
        e = cut_error(np.exp(-fine))
        assert (e.max(1) > 0.8 * 2.0 ** -17).all() and (e.min(1) < -0.8 * 2.0 ** -17).all()
        pairs = [(fine[k, e[k].argmax()], fine[k, e[k].argmin()]) for k in range(3)]
        for t in range(n):
            at, sign = (pairs[(t - 1) // 2][(t - 1) % 2], 1.0 if t % 2 else -1.0) if t else (0.0, 0.0)
            weight[t] = np.exp(-at)
            if fmt == "fp8":
                rows.codes(0, t, -1.0 if t else 0.0, np.float32(at) if t else 1.0)
                rows.codes(1, t, sign, 1.0)
            else:                                                # a key of 20 bits by three features of 8
                k = np.zeros(d)
                for i in range(3):
                    k[i] = np.trunc(-at * 2.0 ** (8 * i + 8)) / 256.0
                    at += k[i] * 2.0 ** (-8 * i)
                assert at == 0.0
                rows.values(0, t, k)
                rows.values(1, t, sign)
        off, size = 0.0, weight[1:].sum()
    want, want_lse = kp.attend(rows.q, rows.held(0), rows.held(1), 1.0)
    np.testing.assert_allclose(want_lse, np.log(weight.sum()), rtol=1e-6)
    out, lse = rows.run()
    tol = (off + (2.0 ** -21 + (n + 4) * 2.0 ** -24) * size) / weight.sum() + 2.0 ** -9 * np.abs(want)
    assert (np.abs(out - want) <= tol).all(), (np.abs(out - want).max(), tol.min())


DTYPES = [kv.KVTC_BF16, kv.KVTC_F32]
LARGEST = float(kp.bf16_value(np.array([0x7F7F], np.uint16))[0])


def spread(d, weights, dtype):
    """Rows whose softmax weights relative to the first token's are 2^weights (d features, one query head): keys of one feature."""
    q = np.zeros(d)
    q[0] = 1.0
    rows = Rows("bf16", d, len(weights), q, dtype, scale=float(np.log(2.0)))
    for t, w in enumerate(weights):
        k = np.zeros(d)
        k[0] = w
        rows.values(0, t, k)
        rows.values(1, t, 0.0)
    return rows


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("weight,value,keeps", [(-300, LARGEST, False), (-300, -LARGEST, False), (-1000, LARGEST, False), (-118, 2.0 ** 120, True), (-110, -2.0 ** 112, True), (-20, 2.0 ** 30, True)])
def test_a_large_value_counts_by_its_weight(dtype, d, weight, value, keeps):
    """A token whose weight is zero in fp32 counts for nothing, whatever its finite value; one of small weight for what it is.  Parts of a probability may be off by 2^-133 each in place of zero."""
    rows = spread(d, [0, weight, -3], dtype)
    rows.values(1, 0, 1.0)
    rows.values(1, 1, value)
    want, want_lse = kp.attend(rows.q, rows.held(0), rows.held(1), rows.scale)
    assert (abs(want[0, 0] - 1 / 1.125) > 0.5) == keeps
    tol, tol_lse = kp.attend_bound(rows.q, rows.held(0), rows.held(1), np.abs(rows.held(0)), np.abs(rows.held(1)), rows.scale, 17 if dtype == kv.KVTC_BF16 else 22, 8 if dtype == kv.KVTC_BF16 else 22)
    out, lse = rows.run()
    assert (np.abs(out - want) <= tol + (2 * 2.0 ** -133 * abs(value) if keeps else 0.0)).all(), (out[0, 0], want[0, 0])
    assert np.abs(lse - want_lse).max() <= tol_lse.max()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("weight", [0, -1, -7, -10.5, -100, -120])
def test_an_infinite_value_stays_one(dtype, d, weight):
    """Whether its probability has parts of zero (powers of two) or not, in its own feature alone; two of opposite signs are none, and nor is one of no weight."""
    rows = spread(d, [0, weight, -300], dtype)
    v = np.ones(d)
    v[3], v[d - 1], v[9] = np.inf, -np.inf, np.inf
    rows.values(1, 1, v)
    v[:] = 1.0
    v[9] = -np.inf
    rows.values(1, 0, v)
    v[:] = 1.0
    v[20] = np.inf
    rows.values(1, 2, v)
    out, lse = rows.run()
    assert np.isposinf(out[0, 3]) and np.isneginf(out[0, d - 1]) and np.isnan(out[0, 9]) and np.isnan(out[0, 20])
    rest = np.delete(out[0], [3, 9, 20, d - 1])
    assert (np.abs(rest - 1.0) <= 2.0 ** -8).all() and np.isfinite(lse).all()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("up", [-105, -97, -60, 60, 100])
def test_fp32_queries_of_any_magnitude(d, up):
    """Queries of 2^up over bf16 pages, the keys as much the other way; scores are as ever, and so is their precision."""
    rng = np.random.default_rng(d + up + 200)
    n = 77
    rows = Rows("bf16", d, n, rng.standard_normal((4, d)) * 2.0 ** up, kv.KVTC_F32, scale=d ** -0.5)
    rows.q[0, ::2] = np.float32(2.0 ** up)                       # (parts of zero)
    for t in range(n):
        rows.values(0, t, rng.standard_normal(d) * 4 * 2.0 ** -up)
        rows.values(1, t, rng.standard_normal(d))
    args = rows.q, rows.held(0), rows.held(1)
    want, want_lse = kp.attend(*args, rows.scale)
    tol, tol_lse = kp.attend_bound(*args, np.abs(args[1]), np.abs(args[2]), rows.scale, 22, 22)
    out, lse = rows.run()
    assert (np.abs(out - want) <= tol).all(), np.abs((out - want) / tol).max()
    assert (np.abs(lse - want_lse) <= tol_lse).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("up,scale_up", [(119, -119), (126, -110), (126, -40), (80, 0), (60, 6), (60, 20), (-60, 60), (-126, 120)])
def test_four_bit_queries_of_any_magnitude(dtype, d, up, scale_up):
    """A feature of 2^up, where all keys are zero, and others whose scores are as ever, with scales of 2^scale_up: the first one, up to 2^86 times the others, takes no bits of theirs."""
    rng = np.random.default_rng(d + up + 200)
    n = 77
    q = rng.standard_normal((4, d)) * 2.0 ** -scale_up
    q[:, 0] = 2.0 ** up
    rows = Rows("int4", d, n, q, dtype, scale=d ** -0.5 * 2.0 ** scale_up)
    for t in range(n):
        for side in range(2):
            k = rng.standard_normal(d) * 4
            if side == 0:
                k[:32] = 1.0                                     # (the first group's range begins at zero)
                k[0] = 0.0
            bytes_, scales = kp.quantise(k.astype(np.float32), "int4")
            r, s = rows.pool.at(t, 0)
            rows.pool.bytes[side][r:r + len(bytes_)], rows.pool.scales[side][s:s + len(scales)] = bytes_, scales
    (kr, ks), (vr, vs) = rows.pool.rows(0, range(n), 0), rows.pool.rows(1, range(n), 0)
    k, v = rows.held(0), rows.held(1)
    assert (k[:, 0] == 0.0).all()
    sizes = kp.sizes(kr, ks, "int4", d)
    sizes[:, 0] = 0.0
    want, want_lse = kp.attend(rows.q, k, v, rows.scale)
    tol, tol_lse = kp.attend_bound(rows.q, k, v, sizes, kp.sizes(vr, vs, "int4", d), rows.scale, 17 if dtype == kv.KVTC_BF16 else 22, 8 if dtype == kv.KVTC_BF16 else 22)
    out, lse = rows.run()
    assert (np.abs(out - want) <= tol).all() and (np.abs(lse - want_lse) <= tol_lse).all()


@pytest.mark.parametrize("fmt,d", [("bf16", 64), ("bf16", 128), ("fp8", 128), ("fp8", 256), ("int4", 64), ("int4", 128), ("int4", 256)])
def test_sums_over_long_rows_are_not_cut(fmt, d):
    """1024 sequences over the same 131072 tokens, positive values: a wave adds up a thousand pieces of 32 tokens.  A piece's sums, in the matrix unit, are off by 128 2^-24 of themselves at most, and
    adding t of them, each rounded to nearest, by t 2^-24, outputs and weights alike; of 4 bits, codes and shifts apart.  Such roundings average out: of t with an error spread evenly over an ulp (2^-24.8 at most),
    of sums that grow evenly, in four waves, sqrt(t / 3) / 2 are left, and five times that is the bound of the features' mean.  (A matrix unit that adds to sums as large cuts off what does not reach their last bit.)"""
    n, n_seqs, page = 131072, 1024, 64
    rng = np.random.default_rng(d)
    pool = Pool(fmt, n // page, page, 1, d)
    for side in range(2):
        x = rng.standard_normal((n, d)).astype(np.float32)
        rows, scales = kp.quantise(np.abs(x) + np.float32(0.25) if side else x, fmt)
        pool.bytes[side][:] = rows.reshape(-1)
        if pool.scale:
            pool.scales[side][:] = scales.reshape(-1)
    cache = pool.upload()
    q = rng.standard_normal((n_seqs, d)).astype(np.float32)
    qd = torch.from_numpy(q).to(DEV)
    pages = torch.from_numpy(np.tile(rng.permutation(n // page).astype(np.int32), (n_seqs, 1))).to(DEV)
    work = Work.get(kv.kvtc_attend_work_bytes(cache, n_seqs, 1, n))
    out, lse = torch.empty_like(qd), torch.empty((n_seqs, 1), device=DEV)
    kv.kvtc_attend(cache, qd, kv.KVTC_F32, n_seqs, 1, d, d, pages, pages.shape[1], torch.full((n_seqs,), n, dtype=torch.int32, device=DEV), n, d ** -0.5, 0, 0, out, lse, work, work.numel())
    torch.cuda.synchronize()
    (kr, ks), (vr, vs) = [pool.rows(side, range(n), 0) for side in range(2)]
    k, v = kp.values(kr, ks, fmt, d), kp.values(vr, vs, fmt, d)
    sizes, t = np.abs(v), n // 32 // 4
    if fmt == "int4":                                            # codes and shifts apart
        shift = np.repeat(np.ascontiguousarray(vs).view(np.float16).astype(np.float64).reshape(n, -1, 2)[..., 0], kp.GROUP, axis=-1)
        sizes = np.abs(shift) + (v - shift)
    off = 2 * (t + 128) * 2.0 ** -24 + 2.0 ** -19                # (2^-19: scores and exponentials)
    for b in (0, 1, 500, 1023):
        want, want_lse = kp.attend(q[b:b + 1], k, v, d ** -0.5)
        size = kp.attend(q[b:b + 1], k, sizes, d ** -0.5)[0]
        err = (out[b].double().cpu().numpy() - want[0]) / size[0]
        assert np.abs(err).max() <= off
        assert abs(err.mean()) <= 5 * np.sqrt(t / 3) / 2 * 2.0 ** -24.8, err.mean()
        assert abs(lse[b, 0].item() - want_lse[0]) <= off + 2.0 ** -21 * abs(want_lse[0])
