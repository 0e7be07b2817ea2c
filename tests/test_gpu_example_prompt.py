"""A prompt in examples/paged_decode.py, behind a restored context and before single tokens: what it sees is what the cache holds."""
import pytest

from test_gpu_example import _example

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("prompt,sequences", [(1, 2), (33, 3), (200, 1)])
def test_a_prompt_behind_a_restored_context(fmt, prompt, sequences):
    r = _example().run(context=700, tokens=20, sequences=sequences, fmt=fmt, prompt=prompt)
    assert r["off_prompt"] < 2.0 ** -8 and r["off"] < 2.0 ** -8  # (the result rounded to bf16, 2^-9 of it in the mean, with as much again for the rest)
    s = r["session"]
    assert s.lengths.tolist() == [700 + max(0, prompt - b) + 20 for b in range(sequences)]
    held = sum(-(-n // 64) for n in s.lengths.tolist())
    assert int(s.n_free.item()) == s.free.numel() - held and len(set(s.pages[s.pages >= 0].tolist())) == held
