"""Places of new tokens (kvtc_cache_place) against the CPU oracle: the same whole numbers."""
import numpy as np
import pytest
import torch

import kvtc_serving as sv
import paper_2511_01815_amd as kv

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


class Case:
    def __init__(self, rng, had, new, page, width, n_free, rows):
        self.had, self.new, self.page, self.rows = np.array(had, np.int64), np.array(new, np.int64), page, rows
        pages = rng.permutation(2 ** 20)[:len(had) * width + max(0, n_free)].astype(np.int32) if len(had) * width + n_free < 2 ** 20 else rng.integers(0, 2 ** 31, len(had) * width + n_free).astype(np.int32)
        self.table = pages[:len(had) * width].reshape(len(had), width).copy()      # (entries that nobody has yet hold numbers too)
        self.free = pages[len(had) * width:]

    def run(self, in_place=False, stream=None):
        n = len(self.had)
        self.dev = dict(had=ints(self.had), new=ints(self.new), table=ints(self.table), free=ints(np.concatenate([self.free, [-7]])), n_free=ints([len(self.free)]),
                        starts=torch.full((n + 2,), 99, dtype=torch.int32, device=DEV), slots=torch.full((self.rows + 1,), 99, dtype=torch.int64, device=DEV),
                        at=torch.full((self.rows + 1,), 99, dtype=torch.int32, device=DEV), status=torch.zeros(1, dtype=torch.int32, device=DEV))
        d = self.dev
        d["out"] = d["had"] if in_place else torch.full((n,), 99, dtype=torch.int32, device=DEV)
        d["left"] = d["n_free"] if in_place else torch.full((1,), 99, dtype=torch.int32, device=DEV)
        kv.kvtc_cache_place(n, d["had"], d["new"], self.page, d["table"], self.table.shape[1], d["free"], d["n_free"], self.rows, d["starts"], d["out"], d["left"], d["slots"], d["at"],
                            d["status"], stream)

    def check(self):
        torch.cuda.synchronize()
        starts, lengths, left, slots, at, table, bad = sv.place(self.had, self.new, self.page, self.table, self.free, self.rows)
        d = {k: t.cpu().numpy() for k, t in self.dev.items()}
        np.testing.assert_array_equal(d["starts"], np.append(starts, 99))
        np.testing.assert_array_equal(d["out"], lengths)
        np.testing.assert_array_equal(d["slots"], np.append(slots, 99))
        np.testing.assert_array_equal(d["at"], np.append(at, 99))
        np.testing.assert_array_equal(d["table"], table)
        assert d["left"][0] == left and d["status"][0] == bad


@pytest.mark.parametrize("page", [1, 16, 20, 64])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seqs,most_new,most_had,padding", [(1, 1, 0, 0), (1, 5000, 33, 7), (64, 1, 3000, 0), (63, 9, 100, 3), (256, 40, 65, 1), (257, 33, 200, 0), (1100, 17, 50, 5), (3, 4100, 90, 40)])
def test_places_are_the_oracles(page, in_place, seqs, most_new, most_had, padding):
    rng = np.random.default_rng(page + seqs)
    had, new = rng.integers(0, most_had + 1, seqs), rng.integers(0, most_new + 1, seqs)
    if seqs == 1:
        new[0] = most_new
    width = -(-(most_new + most_had) // page) + 1
    case = Case(rng, had, new, page, width, int(sum(-(-(h + n) // page) - -(-h // page) for h, n in zip(had, new))) + 3, int(new.sum()) + padding)
    case.run(in_place)
    case.check()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("rows_short", [0, 3, 10 ** 9])
def test_what_has_no_place(in_place, rows_short):
    rng = np.random.default_rng(5)
    n = 300
    had, new = rng.integers(0, 60, n), rng.integers(0, 30, n)
    had[[7, 100]], new[[20, 150]] = -5, -2                          # invalid
    had[40], new[60] = 2 ** 31 - 1, 2 ** 31 - 1                     # beyond any table; sums beyond 31 bits
    for free in (0, 60, 250, 5000):
        total = int(np.clip(new, 0, 10 ** 6).sum())
        case = Case(rng, had, new, 16, 6, free, max(0, total - rows_short))
        case.run(in_place)
        case.check()
    new[60] = 3
    case = Case(rng, had, new, 16, 6, 200, max(0, int(np.clip(new, 0, None).sum()) - rows_short))
    case.run(in_place)
    case.check()


def test_sums_beyond_31_bits_and_many_sequences():
    rng = np.random.default_rng(6)
    new = np.full(2500, 2 ** 31 - 1)
    new[:1200] = rng.integers(0, 3, 1200)
    new[1900:] = 0
    case = Case(rng, rng.integers(0, 9, 2500), new, 4, 4, 4000, 2000)
    case.run()
    case.check()
    case = Case(rng, rng.integers(0, 9, 65536), rng.integers(0, 2, 65536), 4, 4, 40000, 65536)
    case.run()
    case.check()


def test_no_sequences_and_no_rows():
    rng = np.random.default_rng(7)
    for had, new, rows in (([], [], 5), ([], [], 0), ([3, 4], [0, 0], 0), ([3, 4], [0, 0], 4), ([3], [1], 0)):
        case = Case(rng, had, new, 4, 2, 3, rows)
        case.run()
        case.check()


def test_negative_pages_give_no_slot():
    rng = np.random.default_rng(8)
    case = Case(rng, [3, 5], [6, 2], 4, 4, 6, 9)
    case.table[0, 0], case.free[-1] = -1, -3
    case.run()
    case.check()


def test_optional_outputs_and_another_stream():
    rng = np.random.default_rng(9)
    case = Case(rng, [3, 5], [600, 5000], 4, 2000, 3000, 5700)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        case.run(stream=side)
    side.synchronize()
    case.check()
    d = case.dev
    slots = torch.zeros_like(d["slots"])
    kv.kvtc_cache_place(2, ints(case.had), d["new"], 4, ints(case.table), 2000, d["free"], ints([len(case.free)]), 5700, d["starts"], d["out"], d["left"], slots)
    torch.cuda.synchronize()
    assert torch.equal(slots[:5700], d["slots"][:5700])
