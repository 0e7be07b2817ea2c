"""The serving loop of examples/paged_decode.py, small: the attention is that of the cache's own values, and what left the window comes back from its records."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")


def _example():
    spec = importlib.util.spec_from_file_location("paged_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
def test_tokens_attend_to_the_cache_and_the_window_moves_into_records(fmt):
    ex = _example()
    r = ex.run(context=700, tokens=40, sequences=2, fmt=fmt)
    assert r["off"] < 2.0 ** -8                                  # bf16 rounding of the result (2^-9 each), with as much again for the rest
    s = r["session"]
    # 700 tokens restored: 560 stored as they were; then steps of 16 while more than window + 16 are left: up to 740 tokens
    assert s.stored == 560 + 16 * r["steps_stored"] and 128 <= 740 - s.stored < 128 + 16
    last = torch.empty((16, ex.WIDE), dtype=torch.bfloat16, device=ex.DEV)
    at = (s.stored - 16) * s.v.plan.record_bytes
    ex.kv.kvtc_decode(s.v.plan.handle, s.v.records[1, at:], 16 * s.v.plan.record_bytes, 16, last, ex.kv.KVTC_BF16, ex.WIDE)
    k, v = [torch.empty((16, ex.HEADS, ex.D), device=ex.DEV) for _ in range(2)]
    ex.kv.kvtc_cache_read(s.cache, s.slots(1, s.stored - 16, 16), 16, k, v, ex.kv.KVTC_F32, ex.WIDE, ex.D)
    off = float((last.float() - v.view(16, -1)).norm() / v.norm())
    assert off < (0.35 if fmt == "int4" else 0.25), off          # the 16x plan's own error on tensors of its spectrum, and that of 4 bits
