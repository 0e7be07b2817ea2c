"""Attention of many new tokens over the pages of a live cache (kvtc_attend_many) against float64 on the CPU, within the bound of its arithmetic (kvtc_serving.bound)."""
import numpy as np
import pytest
import torch

import kvtc_paged as kp
import kvtc_serving as sv
import paper_2511_01815_amd as kv
from test_gpu_cache import DEV, FORMATS, Pool, host, to_dev

pytestmark = pytest.mark.gpu

NEW = [1, 0, 2, 5, 15, 16, 17, 31, 33, 64, 65, 7, 1, 130, 3]
HAD = [0, 3, 1, 31, 32, 33, 0, 64, 100, 257, 1, 300, 63, 5, 513]


def bits_of(fmt, dtype):
    """Of keys, probabilities and values as they enter their products, and of the result.  fp32 queries: all in fp32 (values rounded once from the cache's).  bf16 queries: over bf16 pages probabilities in
    bf16, else all three in fp16, rounded to nearest: off by half a step at most."""
    if dtype == kv.KVTC_F32:
        return 24, 22, 24, 22
    return (60, 8, 60, 8) if fmt == "bf16" else (11, 11, 11, 8)


class Case:
    """Sequences over a pool filled by the oracle; unused entries of the table are garbage, the rows of tokens that nobody sees too."""

    def __init__(self, rng, fmt, d, heads, group, page, order, new, had, dtype, causal=True, sinks=0, window=0, poison=True, spread=1.0, behind=2, before=0):
        self.fmt, self.d, self.heads, self.group, self.page, self.dtype = fmt, d, heads, group, page, dtype
        self.causal, self.sinks, self.window, self.scale, self.new = causal, sinks, window, d ** -0.5, list(new)
        self.lengths = [n + h for n, h in zip(new, had)] if causal else list(had)
        pages = [-(-n // page) for n in self.lengths]
        n_pages = sum(pages) + 2
        self.pool = Pool(fmt, n_pages, page, heads, d, order)
        if poison:                                               # NaN in 16 bits and in 8, infinite scales; 4-bit headers of infinity
            for side in range(2):
                self.pool.bytes[side][:] = 0xFF
                self.pool.scales[side].view(np.uint8)[:] = np.resize(np.array([0x00, 0x7C], np.uint8), self.pool.scales[side].size) if fmt == "int4" else 0xFF
        order_of = rng.permutation(n_pages)
        self.table = rng.integers(-2 ** 31, 2 ** 31, size=(len(new), max(1, max(pages)) + 2)).astype(np.int32)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + before
        self.rows = int(self.starts[-1]) + behind
        self.q = host(rng.standard_normal((self.rows, heads * group, d)).astype(np.float32) * spread, dtype)
        at = 0
        self.slots = []
        for b, n in enumerate(self.lengths):
            mine = order_of[at:at + pages[b]]
            at += pages[b]
            used = np.zeros(n, bool)
            for i in range(new[b]):
                used[sv.seen(n - new[b] + i, n, causal, sinks, window)] = True
            t = np.nonzero(used)[0]
            self.table[b, np.unique(t // page)] = mine[np.unique(t // page)]
            every = np.arange(n)
            self.slots.append(mine[every // page] * page + every % page if n else np.zeros(0, np.int64))
            for side in range(2):
                x = rng.standard_normal((len(t), heads, d)).astype(np.float32) + rng.standard_normal((heads, d)).astype(np.float32) * 0.5
                x[..., ::29] *= 4
                if len(t):
                    self.pool.put(side, self.slots[b][t], x)
        self.upload()
        self.table_dev = torch.from_numpy(self.table).to(DEV)
        self.starts_dev = torch.from_numpy(self.starts).to(DEV)
        self.lengths_dev = torch.tensor(self.lengths, dtype=torch.int32, device=DEV)
        self.q_dev = to_dev(self.q, dtype)

    def upload(self):
        self.cache = self.pool.upload()

    def run(self, max_tokens=None, lse=True, stream=None, out=None, status=None, work=None):
        hq = self.q.shape[1]
        most = max_tokens or max(1, max(self.lengths))
        need = kv.kvtc_attend_many_work_bytes(self.cache, len(self.new), self.rows, hq, most)
        assert need > 0
        work = torch.zeros(need, dtype=torch.uint8, device=DEV) if work is None else work
        out = out or (torch.full_like(self.q_dev, 5.0), torch.full((self.rows, hq), 5.0, device=DEV))
        status = torch.zeros(1, dtype=torch.int32, device=DEV) if status is None else status
        kv.kvtc_attend_many(self.cache, self.q_dev, self.dtype, len(self.new), self.rows, hq, hq * self.d, self.d, self.starts_dev, self.table_dev, self.table.shape[1], self.lengths_dev, most,
                            self.scale, self.causal, self.sinks, self.window, out[0], out[1] if lse else None, work, work.numel(), status, stream)
        return out[0], out[1], status

    def check(self, out, lse, only=None, gone=None, rows=None):
        """gone: {sequence: tokens that are not seen after all}; rows: of each sequence, which (all)."""
        out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        for b, n in enumerate(self.new):
            if only is not None and b not in only:
                continue
            for h in range(self.heads):
                (kr, ks), (vr, vs) = self.pool.rows(0, self.slots[b], h), self.pool.rows(1, self.slots[b], h)
                k, v = kp.values(kr, ks, self.fmt, self.d), kp.values(vr, vs, self.fmt, self.d)
                at = slice(h * self.group, (h + 1) * self.group)
                for i in range(n) if rows is None else rows:
                    t = sv.seen(self.lengths[b] - n + i, self.lengths[b], self.causal, self.sinks, self.window)
                    if gone and b in gone:
                        t = t[~np.isin(t, gone[b])]
                    r = self.starts[b] + i
                    want, want_lse = kp.attend(self.q[r, at], k[t], v[t], self.scale)
                    tol, tol_lse = sv.bound(self.q[r, at], k[t], v[t], self.scale, *bits_of(self.fmt, self.dtype))
                    assert (np.abs(out[r, at] - want) <= tol).all(), (b, h, i, np.abs(out[r, at] - want).max(), tol.min())
                    if len(t) == 0:
                        assert (out[r, at] == 0).all() and np.isneginf(lse[r, at]).all()
                    else:
                        assert (np.abs(lse[r, at] - want_lse) <= tol_lse).all(), (b, h, i, np.abs(lse[r, at] - want_lse).max(), tol_lse.min())
        outside = np.ones(self.rows, bool)
        outside[self.starts[0]:self.starts[-1]] = False
        assert (out[outside] == 5.0).all() and (lse[outside] == 5.0).all()      # rows of no sequence stay as they were


SHAPES = [(128, 2, 4, 64, "heads"), (128, 2, 5, 16, "tokens"), (64, 3, 1, 20, "heads"), (256, 1, 8, 32, "tokens"), (128, 1, 16, 1, "heads"), (64, 1, 17, 128, "tokens"), (256, 2, 2, 7, "slab")]


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d,heads,group,page,order", SHAPES)
def test_lengths_around_every_edge(fmt, dtype, d, heads, group, page, order):
    case = Case(np.random.default_rng(d + group + page), fmt, d, heads, group, page, order, NEW, HAD, dtype, before=group % 3)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_a_whole_group_of_many_query_heads(fmt, dtype):
    """More query heads to a KV head than an item has rows."""
    case = Case(np.random.default_rng(11), fmt, 64, 1, 300, 32, "heads", [3, 1, 2], [40, 0, 70], dtype)
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("sinks,window", [(4, 128), (0, 1), (0, 33), (33, 31), (1, 64), (500, 20), (7, 10 ** 9), (70, 65)])
def test_sinks_and_windows(fmt, dtype, sinks, window):
    case = Case(np.random.default_rng(sinks + window), fmt, 64, 2, 3, 16, "tokens", [40, 1, 0, 90, 3, 130], [0, 700, 9, 66, 129, 300], dtype, True, sinks, window)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_tokens_of_another_length(fmt, dtype, d):
    """Not causal: every row sees all tokens of a sequence of any length, none among them."""
    case = Case(np.random.default_rng(d), fmt, d, 2, 2, 20, "heads", [3, 70, 1, 5, 33], [0, 1, 65, 200, 31], dtype, causal=False)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    case.check(out, lse)


def test_more_new_tokens_than_a_sequence_has():
    """Rows at positions before the sequence's first token see nothing."""
    case = Case(np.random.default_rng(12), "bf16", 64, 1, 2, 16, "heads", [5, 9], [0, 3], kv.KVTC_BF16)
    case.lengths_dev = torch.tensor([2, 12], dtype=torch.int32, device=DEV)
    out, lse, _ = case.run(max_tokens=12)
    torch.cuda.synchronize()
    case.check(out, lse, only=[1])
    assert bool((out[:3] == 0).all()) and bool(torch.isneginf(lse[:3]).all())
    case.lengths[0] = 2
    case.check(out, lse)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d,page", [(128, 64), (64, 24), (256, 16)])
def test_long_contexts_are_split_and_joined(fmt, dtype, d, page):
    """Few rows over long contexts: an item's tiles are shared by many workgroups; next to it short ones."""
    case = Case(np.random.default_rng(page), fmt, d, 1, 4, page, "heads", [6, 0, 3, 1, 2], [9001, 0, 3, 4000, 0], dtype)
    first = case.run()
    again = case.run()
    torch.cuda.synchronize()
    case.check(first[0], first[1])
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    wide = case.run(max_tokens=case.page * case.table.shape[1])      # a bound that says little
    torch.cuda.synchronize()
    case.check(wide[0], wide[1])
    none = case.run(lse=False)
    torch.cuda.synchronize()
    assert torch.equal(none[0], first[0]) and bool((none[1] == 5.0).all())


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_prompt_of_many_tokens(fmt, dtype, d):
    case = Case(np.random.default_rng(13), fmt, d, 2, 3, 16, "tokens", [700, 1, 450], [0, 0, 333], dtype)
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse, rows=None if d == 64 else range(0, 450, 7), only=None if d == 64 else [0, 2])


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("few", [False, True])
def test_invalid_sequences_and_pages_are_reported_and_hurt_nobody_else(fmt, dtype, few):
    rng = np.random.default_rng(4)
    new, had = ([4, 3, 2, 5, 1], [40, 100, 70, 195, 60]) if few else ([60, 70, 40, 90, 30], [40, 100, 70, 110, 60])
    case = Case(rng, fmt, 128, 2, 4, 16, "heads", new, had, dtype)
    n_pages = case.pool.n_pages
    table = case.table.copy()
    table[3, 5], table[3, 7] = n_pages, -1                           # tokens 80..95 and 112..127 of sequence 3
    case.table_dev = torch.from_numpy(table).to(DEV)
    bad = torch.tensor(case.lengths, dtype=torch.int32, device=DEV)
    bad[1], bad[4] = -3, 201
    case.lengths_dev = bad
    out, lse, status = case.run(max_tokens=200)
    torch.cuda.synchronize()
    assert int(status.item()) == 2
    gone = {3: np.r_[80:96, 112:128]}
    case.check(out, lse, only=[0, 2, 3], gone=gone)
    for b in (1, 4):
        rows = slice(int(case.starts[b]), int(case.starts[b + 1]))
        assert bool((out[rows] == 0).all()) and bool(torch.isneginf(lse[rows]).all())
    case.lengths_dev = torch.tensor(case.lengths, dtype=torch.int32, device=DEV)
    out, lse, status = case.run(max_tokens=max(case.lengths))
    torch.cuda.synchronize()
    assert int(status.item()) == 4
    case.check(out, lse, gone=gone)
    # starts that are not ascending or leave the batch: those sequences' rows stay, the others are as they were
    starts = case.starts.copy()
    starts[-1] = case.rows + 1
    case.starts_dev = torch.from_numpy(starts).to(DEV)
    out, lse, status = case.run(max_tokens=max(case.lengths))
    torch.cuda.synchronize()
    assert int(status.item()) == 4
    case.check(out, lse, only=[0, 1, 2])
    assert bool((out[int(case.starts[4]):] == 5.0).all())


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_infinities_and_nan_reach_only_rows_that_see_them(fmt, dtype, d):
    """A token whose values (or keys) are NaN or infinite, behind some rows' positions and before others'."""
    rng = np.random.default_rng(14)
    case = Case(rng, fmt, d, 1, 3, 16, "heads", [50, 70], [30, 0], dtype)
    spoilt = {0: 47, 1: 33}                                          # tokens; the rows of positions before these must not change
    for b, t in spoilt.items():
        r, s = case.pool.at(int(case.slots[b][t]), 0)
        side = 1 if b == 0 else 0
        if fmt == "bf16":
            case.pool.bytes[side][r:r + 2 * d] = np.full(d, 0x7F80 if b == 0 else 0x7FC0, np.uint16).view(np.uint8)
        elif fmt == "fp8":
            case.pool.bytes[side][r:r + d] = 0x7F
        else:
            case.pool.scales[side][s:s + d // 8] = np.full(d // 16, 0x7C00, np.uint16).view(np.uint8)
    case.upload()
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    for b, t in spoilt.items():
        first = int(case.starts[b])
        clean = t - (case.lengths[b] - case.new[b])                  # rows before the token
        case.check(out, lse, only=[b], rows=range(clean))
        seeing = out[first + clean:int(case.starts[b + 1])].float()
        assert not bool(torch.isfinite(seeing).any())


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_scores_of_large_spread(dtype):
    """Scores of hundreds in either direction, and a key of minus infinity along the query."""
    rng = np.random.default_rng(5)
    case = Case(rng, "bf16", 64, 1, 4, 32, "heads", [40, 3], [300, 700], dtype, spread=30.0)
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse)
    case.q[..., 0] = np.abs(case.q[..., 0]) + 0.5
    case.q = host(case.q, dtype)                                     # (what the kernel gets)
    case.q_dev = to_dev(case.q, dtype)
    gone = {0: np.array([33]), 1: np.array([64])}
    for b, t in gone.items():
        r = case.pool.at(int(case.slots[b][t[0]]), 0)[0]
        case.pool.bytes[0][r:r + 2] = np.array([0xFF80], np.uint16).view(np.uint8)
    case.upload()
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse, gone=gone)


@pytest.mark.parametrize("scale", [0.0, -0.11, 1e-30])
@pytest.mark.parametrize("fmt", list(FORMATS))
def test_scales_of_any_sign(fmt, scale):
    case = Case(np.random.default_rng(15), fmt, 128, 1, 2, 16, "heads", [20, 3], [0, 100], kv.KVTC_BF16)
    case.scale = scale
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("size", [1e-30, 1e15])
def test_queries_of_any_magnitude(fmt, size):
    """The product with the scale is what it was: only the queries' exponents differ."""
    rng = np.random.default_rng(16)
    case = Case(rng, fmt, 128, 1, 2, 16, "heads", [20, 3], [0, 100], kv.KVTC_BF16)
    case.q = host(case.q * np.float32(size), kv.KVTC_BF16)
    case.q_dev = to_dev(case.q, kv.KVTC_BF16)
    case.scale = float(np.float32(128 ** -0.5 / size))
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse)


@pytest.mark.parametrize("fmt", ["fp8", "int4"])
def test_rows_of_very_different_scales(fmt):
    """8- and 4-bit rows whose scales differ by 2^20 from token to token."""
    rng = np.random.default_rng(17)
    case = Case(rng, fmt, 128, 1, 2, 16, "heads", [40, 3], [30, 300], kv.KVTC_BF16)
    for side in range(2):
        for b in range(2):
            x = rng.standard_normal((case.lengths[b], 1, 128)).astype(np.float32)
            x *= np.exp2(rng.integers(-10, 1, case.lengths[b])).astype(np.float32)[:, None, None] * (1.0 if side == 0 else 2.0 ** -5)
            case.pool.put(side, case.slots[b], x)
    case.upload()
    out, lse, _ = case.run()
    torch.cuda.synchronize()
    case.check(out, lse)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("new,had", [([1, 2, 5], [0, 3, 0]), ([33, 1, 64], [0, 700, 200]), ([130], [1500])])
def test_sums_over_four_bits_are_those_of_the_caches_own_keys(d, new, had):
    """Where bf16 queries meet codes, lse is still fp32's: no key is rounded.  A score is the sum over groups of scale * (codes . q) + shift * (sum of q).  Sums of 32 products, two terms to each of d / 32 <= 8 groups and
    three parts of the sum of q, all in fp32, are off by (32 + 16 + 3) 2^-24 < 2^-18 of M = sum of |q| (|shift| + 15 scale) <= 3 sum of |q| max |k| over a group, whose least and largest values have the codes 0 and 15; lse
    is off by no more than its largest score, and by its own rounding and that of the sum: 2^-18 (1 + |lse|)."""
    case = Case(np.random.default_rng(d + len(new)), "int4", d, 2, 3, 16, "heads", new, had, kv.KVTC_BF16)
    out, lse, status = case.run()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    lse = lse.double().cpu().numpy()
    for b, n in enumerate(new):
        for h in range(2):
            k = kp.values(*case.pool.rows(0, case.slots[b], h), "int4", d)
            group = np.repeat(np.abs(k).reshape(len(k), d // 32, 32).max(-1), 32, axis=1)
            for i in range(n):
                r, t, at = case.starts[b] + i, case.lengths[b] - n + i + 1, slice(3 * h, 3 * h + 3)
                s = case.scale * (case.q[r, at].astype(np.float64) @ k[:t].T)
                want = np.log(np.exp(s - s.max(-1, keepdims=True)).sum(-1)) + s.max(-1)
                most = 1.02 * 3 * case.scale * (np.abs(case.q[r, at]) @ group[:t].T).max(-1)
                assert (np.abs(lse[r, at] - want) <= 2.0 ** -18 * (most + 1 + np.abs(want))).all(), (b, h, i, np.abs(lse[r, at] - want).max(), most)


def test_queries_inside_a_fused_projection_and_heads_first():
    rng = np.random.default_rng(6)
    case = Case(rng, "int4", 128, 2, 4, 64, "heads", [33, 1, 5], [333, 64, 0], kv.KVTC_BF16, behind=0)
    n, hq, d = case.q.shape
    want = case.run()
    torch.cuda.synchronize()
    case.check(want[0], want[1])
    whole = torch.full((n, hq * d + 4 * d), float("nan"), dtype=torch.bfloat16, device=DEV)
    whole[:, 2 * d:2 * d + hq * d] = case.q_dev.view(n, -1)
    first = case.q_dev.transpose(0, 1).contiguous()
    work = torch.zeros(kv.kvtc_attend_many_work_bytes(case.cache, 3, n, hq, 366), dtype=torch.uint8, device=DEV)
    for q, ts, hs in ((whole[:, 2 * d:].data_ptr(), whole.shape[1], d), (first, d, n * d)):
        out, lse = torch.empty((n, hq, d), dtype=torch.bfloat16, device=DEV), torch.empty((n, hq), device=DEV)
        kv.kvtc_attend_many(case.cache, q, kv.KVTC_BF16, 3, n, hq, ts, hs, case.starts_dev, case.table_dev, case.table.shape[1], case.lengths_dev, 366, case.scale, True, 0, 0, out, lse, work,
                            work.numel())
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
def test_a_pool_beyond_4_gib(dtype):
    heads, d, page = 8, 128, 64
    n_pages = (5 << 30) // (page * heads * d * 2)
    k, v = [torch.full((n_pages, heads, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache = kv.cache(kv.KVTC_CACHE_BF16, n_pages, page, heads, d, k, v, page * heads * d * 2, page * d * 2, d * 2)
    pages = [n_pages - 1, 0, n_pages - 2]
    rng = np.random.default_rng(7)
    x = [host(rng.standard_normal((3, heads, page, d)).astype(np.float32), kv.KVTC_BF16) for _ in range(2)]
    for i, p in enumerate(pages):
        k[p], v[p] = to_dev(x[0][i], kv.KVTC_BF16), to_dev(x[1][i], kv.KVTC_BF16)
    q = host(rng.standard_normal((5, heads, d)).astype(np.float32), dtype)
    qd = to_dev(q, dtype)
    work = torch.zeros(kv.kvtc_attend_many_work_bytes(cache, 1, 5, heads, 180), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(qd), torch.empty((5, heads), device=DEV)
    kv.kvtc_attend_many(cache, qd, dtype, 1, 5, heads, heads * d, d, torch.tensor([0, 5], dtype=torch.int32, device=DEV), torch.tensor([pages], dtype=torch.int32, device=DEV), 3,
                        torch.tensor([180], dtype=torch.int32, device=DEV), 180, d ** -0.5, True, 0, 0, out, lse, work, work.numel())
    torch.cuda.synchronize()
    for h in range(heads):
        kh, vh = [np.concatenate(a[:, h])[:180] for a in x]
        for i in range(5):
            want, want_lse = kp.attend(q[i, h:h + 1], kh[:176 + i], vh[:176 + i], d ** -0.5)
            tol, tol_lse = sv.bound(q[i, h:h + 1], kh[:176 + i], vh[:176 + i], d ** -0.5, *bits_of("bf16", dtype))
            assert (np.abs(out[i, h:h + 1].float().cpu().numpy() - want) <= tol).all() and np.abs(lse[i, h].item() - want_lse[0]) <= tol_lse[0]


def test_one_row_to_a_sequence_is_a_decode_step():
    rng = np.random.default_rng(18)
    case = Case(rng, "fp8", 128, 4, 4, 32, "heads", [1] * 9, [0, 1, 31, 32, 700, 3000, 5, 64, 127], kv.KVTC_BF16, behind=0)
    out, lse, _ = case.run()
    work = torch.zeros(kv.kvtc_attend_work_bytes(case.cache, 9, 16, 3001), dtype=torch.uint8, device=DEV)
    want, want_lse = torch.empty_like(out), torch.empty_like(lse)
    kv.kvtc_attend(case.cache, case.q_dev, kv.KVTC_BF16, 9, 16, 16 * 128, 128, case.table_dev, case.table.shape[1], case.lengths_dev, 3001, case.scale, 0, 0, want, want_lse, work, work.numel())
    torch.cuda.synchronize()
    case.check(out, lse)
    assert float((lse - want_lse).abs().max()) < 2e-2 and float((out.float() - want.float()).norm() / want.float().norm()) < 2.0 ** -8


def test_calls_that_share_a_workspace():
    """Large and small calls in turn on one stream, each as alone."""
    rng = np.random.default_rng(19)
    cases = [Case(rng, "bf16", 64, 1, 4, 16, "heads", [3, 2], [5000, 100], kv.KVTC_BF16), Case(rng, "fp8", 128, 2, 2, 16, "heads", [1, 4], [900, 2000], kv.KVTC_BF16),
             Case(rng, "bf16", 64, 2, 1, 16, "heads", [5], [3000], kv.KVTC_F32)]
    alone = [c.run() for c in cases]
    most = max(kv.kvtc_attend_many_work_bytes(c.cache, len(c.new), c.rows, c.q.shape[1], max(c.lengths)) for c in cases)
    work = torch.zeros(most, dtype=torch.uint8, device=DEV)
    got = [[c.run(work=work) for c in cases] for _ in range(3)]
    torch.cuda.synchronize()
    for turn in got:
        for g, a in zip(turn, alone):
            assert torch.equal(g[0], a[0]) and torch.equal(g[1], a[1])


def test_a_workspace_shared_with_single_tokens():
    """kvtc_attend counts on zeros that it left; calls of kvtc_attend_many in between, whatever else the workspace holds, do not change what either gives."""
    rng = np.random.default_rng(23)
    many = [Case(rng, "fp8", 128, 2, 4, 16, "heads", [5, 3], [6000, 300], kv.KVTC_BF16), Case(rng, "bf16", 64, 2, 1, 16, "heads", [4], [2500], kv.KVTC_F32)]
    one = Case(rng, "bf16", 128, 2, 4, 16, "heads", [1] * 3, [9000, 40, 2000], kv.KVTC_BF16, before=0, behind=0)
    hq, most = one.q.shape[1], max(one.lengths)
    need = max([kv.kvtc_attend_many_work_bytes(c.cache, len(c.new), c.rows, c.q.shape[1], max(c.lengths)) for c in many] + [kv.kvtc_attend_work_bytes(one.cache, 3, hq, most)])
    work = torch.zeros(need, dtype=torch.uint8, device=DEV)

    def step():
        out, lse = torch.empty_like(one.q_dev), torch.empty((3, hq), device=DEV)
        kv.kvtc_attend(one.cache, one.q_dev, kv.KVTC_BF16, 3, hq, hq * one.d, one.d, one.table_dev, one.table.shape[1], one.lengths_dev, most, one.scale, 0, 0, out, lse, work, work.numel())
        return out, lse

    want_many, want = [c.run() for c in many], step()
    for _ in range(3):
        for c, w in zip(many, want_many):
            got = c.run(work=work)
            assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
            again = step()
            assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    garbage = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)      # of any contents, for kvtc_attend_many
    for c, w in zip(many, want_many):
        got = c.run(work=garbage)
        assert torch.equal(got[0], w[0]) and torch.equal(got[1], w[1])
    assert (garbage[:4096] == 0xFF).all()


def test_calls_at_once_on_two_streams():
    """Each with a workspace of its own."""
    rng = np.random.default_rng(29)
    cases = [Case(rng, "int4", 128, 2, 4, 16, "heads", [6, 3], [5000, 300], kv.KVTC_BF16), Case(rng, "bf16", 128, 2, 4, 20, "tokens", [40, 33], [1500, 64], kv.KVTC_BF16)]
    alone = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(8):
        for g, c, s in zip(got, cases, streams):
            with torch.cuda.stream(s):
                g.append(c.run(stream=s.cuda_stream))
    torch.cuda.synchronize()
    for g, a in zip(got, alone):
        assert all(torch.equal(x[0], a[0]) and torch.equal(x[1], a[1]) and int(x[2].item()) == 0 for x in g)


def test_places_positions_tokens_and_attention_under_capture():
    """A recorded step -- places, rotations of queries and keys, tokens written, attention over them and over a shared prefix, joined -- with new inputs in the same buffers, as eager calls, on every replay; and the
    eager calls against the oracle's values."""
    rng = np.random.default_rng(20)
    heads, group, d, page, seqs, rows = 2, 4, 128, 16, 5, 70
    hq, n_pages, width = heads * group, 120, 40
    had, new = [100, 0, 33, 16, 250], [20, 17, 1, 16, 3]             # 57 rows, 13 of padding
    form, theta = kv.rope_form(d, kv.ROPE_HALF, 500000.0, kv.ROPE_SCALE_BANDS, 8.0, 8192, 1.0, 4.0), sv.frequencies(d, 500000.0, "bands", 8.0, 8192, 1.0, 4.0)
    k, v = [torch.randn((n_pages, heads, page, d), device=DEV).to(torch.bfloat16) for _ in range(2)]
    cache = kv.cache(kv.KVTC_CACHE_BF16, n_pages, page, heads, d, k, v, heads * page * d * 2, page * d * 2, d * 2)
    order = rng.permutation(n_pages).astype(np.int32)
    prefix = torch.from_numpy(np.concatenate([order[:5], np.full(14, -1, np.int32)])).to(DEV)      # 75 tokens that all rows see as well, in pages of their own
    table = np.full((seqs, width), -1, np.int32)
    at = 5
    for b in range(seqs):
        n = -(-had[b] // page)
        table[b, :n] = order[at:at + n]
        at += n
    free = order[at:]
    keep = dict(had=torch.tensor(had, dtype=torch.int32, device=DEV), new=torch.tensor(new, dtype=torch.int32, device=DEV), free=torch.from_numpy(free.copy()).to(DEV),
                n_free=torch.tensor([len(free)], dtype=torch.int32, device=DEV), prefix_starts=torch.tensor([0, rows], dtype=torch.int32, device=DEV),
                prefix_length=torch.tensor([75], dtype=torch.int32, device=DEV), table=torch.from_numpy(table).to(DEV))
    inputs = [torch.randn((rows, hq + 2 * heads, d), device=DEV).to(torch.bfloat16) for _ in range(2)]
    x = inputs[0].clone()
    work = [torch.zeros(kv.kvtc_attend_many_work_bytes(cache, s, rows, hq, 300), dtype=torch.uint8, device=DEV) for s in (seqs, 1)]

    def buffers():
        return dict(starts=torch.zeros(seqs + 1, dtype=torch.int32, device=DEV), lengths=torch.zeros(seqs, dtype=torch.int32, device=DEV), left=torch.zeros(1, dtype=torch.int32, device=DEV),
                    slots=torch.zeros(rows, dtype=torch.int64, device=DEV), at=torch.zeros(rows, dtype=torch.int32, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV),
                    turned=torch.zeros((rows, hq + heads, d), dtype=torch.bfloat16, device=DEV), own=torch.zeros((rows, hq, d), dtype=torch.bfloat16, device=DEV),
                    own_lse=torch.zeros((rows, hq), device=DEV), shared=torch.zeros((rows, hq, d), dtype=torch.bfloat16, device=DEV), shared_lse=torch.zeros((rows, hq), device=DEV),
                    out=torch.zeros((rows, hq, d), device=DEV), lse=torch.zeros((rows, hq), device=DEV))

    def step(b):
        kv.kvtc_cache_place(seqs, keep["had"], keep["new"], page, keep["table"], width, keep["free"], keep["n_free"], rows, b["starts"], b["lengths"], b["left"], b["slots"], b["at"], b["status"])
        wide = (hq + 2 * heads) * d
        kv.kvtc_rope_scaled(x, b["turned"], kv.KVTC_BF16, rows, hq + heads, d, wide, d, (hq + heads) * d, d, b["at"], 0, form)
        keys, values = b["turned"][:, hq:].contiguous(), x[:, hq + heads:].contiguous()
        kv.kvtc_cache_write(cache, keys, values, kv.KVTC_BF16, rows, heads * d, d, b["slots"], b["status"])
        kv.kvtc_attend_many(cache, b["turned"], kv.KVTC_BF16, seqs, rows, hq, (hq + heads) * d, d, b["starts"], keep["table"], width, b["lengths"], 300, d ** -0.5, True, 0, 0, b["own"], b["own_lse"],
                            work[0], work[0].numel(), b["status"])
        kv.kvtc_attend_many(cache, b["turned"], kv.KVTC_BF16, 1, rows, hq, (hq + heads) * d, d, keep["prefix_starts"], prefix, 19, keep["prefix_length"], 300, d ** -0.5, False, 0, 0, b["shared"],
                            b["shared_lse"], work[1], work[1].numel(), b["status"])
        kv.kvtc_attend_join([b["own"], b["shared"]], [b["own_lse"], b["shared_lse"]], kv.KVTC_BF16, rows, hq, d, b["out"], kv.KVTC_F32, b["lse"])

    before = [k.clone(), v.clone()]
    eager = []
    for i in range(2):
        k.copy_(before[0]), v.copy_(before[1]), x.copy_(inputs[i])
        b = buffers()
        step(b)
        torch.cuda.synchronize()
        assert int(b["status"].item()) == 0
        eager.append({n: t.clone() for n, t in b.items()})
    # the oracle, on the last inputs
    starts, lengths, left, slots, positions, grown, bad = sv.place(had, new, page, table, free, rows)
    assert bad == 0 and left == int(b["left"].item()) and (lengths == b["lengths"].cpu().numpy()).all() and (b["slots"].cpu().numpy() == slots).all() and (b["at"].cpu().numpy() == positions).all() and (keep["table"].cpu().numpy() == grown).all()
    turned = sv.rope_scaled(x[:, :hq + heads].double().cpu().numpy(), positions, theta)
    assert np.abs(b["turned"].double().cpu().numpy() - turned).max() <= 2.0 ** -8 * np.abs(turned).max() + 1e-5
    q, kk, vv = b["turned"].double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy()
    for s in range(seqs):
        for i in range(0, new[s], 3):
            r, n = starts[s] + i, had[s] + i + 1
            t = np.arange(n)
            for h in range(heads):
                keys = np.concatenate([kk[grown[s][t // page], h, t % page], kk[order[:5]][:, h].reshape(-1, d)[:75]])
                vals = np.concatenate([vv[grown[s][t // page], h, t % page], vv[order[:5]][:, h].reshape(-1, d)[:75]])
                mine = slice(h * group, h * group + group)
                want, want_lse = kp.attend(q[r, mine], keys, vals, d ** -0.5)
                tol, tol_lse = sv.bound(q[r, mine], keys, vals, d ** -0.5, *bits_of("bf16", kv.KVTC_BF16))
                # (each part is rounded to bf16, of its own size: 2^-8 of the parts' sum of p |v| at most)
                p = np.exp(d ** -0.5 * (q[r, mine] @ keys.T) - want_lse[:, None])
                assert (np.abs(b["out"][r, mine].double().cpu().numpy() - want) <= tol + 2.0 ** -8 * (p @ np.abs(vals))).all()
                assert (np.abs(b["lse"][r, mine].double().cpu().numpy() - want_lse) <= tol_lse + 2.0 ** -20).all()
    got = buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(got)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for n, t in got.items():
        assert torch.equal(t, eager[1][n]), n
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    for i in (0, 1, 0, 1):
        k.copy_(before[0]), v.copy_(before[1]), x.copy_(inputs[i])
        for t in got.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for n, t in got.items():
            assert torch.equal(t, eager[i][n]), f"{n}: replay with input {i} differs from the eager calls"
        step(buffers())                                              # the program's own eager work between replays
        torch.cuda.synchronize()
