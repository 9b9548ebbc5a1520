"""examples/decode_samples.py with a single sample, which is not forked and does not end early."""
import pytest

import test_gpu_example

pytestmark = pytest.mark.gpu


def test_one_sample():
    test_gpu_example.test_decode_samples(dict(tokens=900, samples=1, steps=5, page=32))
