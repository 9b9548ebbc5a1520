"""examples/decode_samples.py at a small size: prefill, cache, fork, graph-captured decoding,
freeing and compaction together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kw", [dict(tokens=1500, samples=5, steps=9, page=16),
                                dict(tokens=2048, samples=12, steps=4, heads=16, kv_heads=2)])
def test_decode_samples(kw):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location(
        "decode_samples", os.path.join(ROOT, "examples", "decode_samples.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    # outputs are means of unit normals over thousands of tokens, a few tenths at most: one bf16
    # rounding of them is below 2e-3
    assert example.run(**kw) <= 2e-3
