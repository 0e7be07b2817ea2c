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


@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("n_seqs,had", [(3, 9000), (513, 40), (1030, 40), (600, 3000)])
def test_nothing_is_written_behind_the_workspace(dtype, n_seqs, had):
    """One sequence with a long context: parts, and where sequences are many, their starts in order as well."""
    case = Case(np.random.default_rng(n_seqs), "int4", 64, 1, 2, 16, "heads", [3] + [1] * (n_seqs - 1), [had] + [5] * (n_seqs - 1), dtype)
    need = kv.kvtc_attend_many_work_bytes(case.cache, n_seqs, case.rows, 2, max(case.lengths))
    whole = torch.full((need + 65536,), 0xA5, dtype=torch.uint8, device=DEV)
    out, lse, status = case.run(work=whole[:need])
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and bool((whole[need:] == 0xA5).all()) and bool((whole[:4096] == 0xA5).all())
    case.check(out, lse, only={0, 1, n_seqs // 2, n_seqs - 1})
    with pytest.raises(kv.KvtcError, match="KVTC_E_SMALL"):
        case.run(work=whole[:need - 1])


def test_many_sequences_under_capture():
    """Starts that change between replays."""
    rng = np.random.default_rng(31)
    n_seqs = 700
    case = Case(rng, "bf16", 64, 1, 2, 16, "heads", [int(n) for n in rng.integers(1, 4, n_seqs)], [int(n) for n in rng.integers(0, 40, n_seqs)], kv.KVTC_BF16)
    spoilt = case.starts.copy()
    spoilt[[20, 300, 650]] = -5, 3, 1 << 30
    kinds = [torch.from_numpy(s).to(DEV) for s in (case.starts, spoilt)]
    most = max(case.lengths)
    work = torch.zeros(kv.kvtc_attend_many_work_bytes(case.cache, n_seqs, case.rows, 2, most), dtype=torch.uint8, device=DEV)
    out, status = (torch.empty_like(case.q_dev), torch.empty((case.rows, 2), device=DEV)), torch.zeros(1, dtype=torch.int32, device=DEV)

    def clear():
        out[0].fill_(5.0), out[1].fill_(5.0), status.zero_()

    eager = []
    for starts in kinds:
        case.starts_dev.copy_(starts)
        clear()
        case.run(out=out, status=status, work=work)
        torch.cuda.synchronize()
        eager.append([t.clone() for t in (*out, status)])
    assert [int(e[2].item()) for e in eager] == [sv.served(s, case.rows)[1] for s in (case.starts, spoilt)] == [0, 20]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.run(out=out, status=status, work=work, stream=torch.cuda.current_stream().cuda_stream)
    for i in (0, 1, 1, 0):
        case.starts_dev.copy_(kinds[i])
        clear()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*out, status), eager[i])), i
        case.run()                                                   # the program's own eager work between replays
        torch.cuda.synchronize()
