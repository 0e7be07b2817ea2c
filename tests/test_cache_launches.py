"""Large writes and reads of the live cache are several launches: how large one may be (CPU), and that rows, slots and reported tokens are right across their seams (GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2511_01815_amd as kv
from test_gpu_cache import DEV, FORMATS, Pool, features, to_dev


def test_a_launch_is_one_that_the_runtime_takes():
    """A row is d / 8 work-items, in workgroups of 256; a launch has fewer than 2^32 of them, and no fewer tokens than that leaves room for."""
    for d in (64, 128, 256):
        for heads in (1, 2, 3, 7, 8, 40, 127, 1023, 1024):
            most = kv.lib().kvtc_host_cache_launch_tokens(heads, d)
            items = [-(-n * heads * (d // 8) // 256) * 256 for n in (most, most + 1)]
            assert most >= 1 and items[0] < 1 << 32 and items[1] >= (1 << 32) - 256 - 256 * heads, (d, heads, most)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [kv.KVTC_BF16, kv.KVTC_F32])
@pytest.mark.parametrize("d,heads,page,order,each", [(64, 3, 20, "tokens", 37), (128, 8, 16, "heads", 64), (256, 2, 7, "slab", 1)])
def test_seams_between_launches(fmt, dtype, d, heads, page, order, each):
    rng = np.random.default_rng(d + each)
    n, n_pages = 203, -(-203 // page) + 2
    slots = rng.permutation(n_pages * page)[:n].astype(np.int64)
    slots[[3, 130]] = -1
    slots[[150, 199]] = n_pages * page + 1
    slots = torch.from_numpy(slots).to(DEV)
    heads_major = order == "slab"
    shape = (heads, n, d) if heads_major else (n, heads, d)
    ts, hs = (d, n * d) if heads_major else (heads * d, d)
    x = [to_dev(features(rng, shape), dtype) for _ in range(2)]
    pools = [Pool(fmt, n_pages, page, heads, d, order) for _ in range(2)]
    caches = [p.upload() for p in pools]
    outs = [[torch.full(shape, 3.0, dtype=x[0].dtype, device=DEV) for _ in range(2)] for _ in range(2)]
    status = torch.zeros(4, dtype=torch.int32, device=DEV)
    kv.kvtc_cache_write(caches[0], x[0], x[1], dtype, n, ts, hs, slots, status[0:])
    kv.kvtc_cache_read(caches[0], slots, n, outs[0][0], outs[0][1], dtype, ts, hs, status[1:])
    stream = torch.cuda.current_stream().cuda_stream
    for write, (k, v), s in ((1, x, status[2:]), (0, outs[1], status[3:])):
        assert kv.lib().kvtc_test_cache_tokens(write, C.byref(caches[1]), k.data_ptr(), v.data_ptr(), dtype, n, ts, hs, slots.data_ptr(), s.data_ptr(), each, stream) == 0
    torch.cuda.synchronize()
    assert status.cpu().tolist() == [151] * 4
    for side in range(2):
        assert torch.equal(pools[0].dev[side], pools[1].dev[side]) and torch.equal(pools[0].dev_scales[side], pools[1].dev_scales[side])
        assert torch.equal(outs[0][side], outs[1][side])
