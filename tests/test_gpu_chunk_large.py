"""Values near the largest of their type: a mean of many is what they are, and no sum on the way to it
passes float32."""
import numpy as np
import pytest

from cache_model import bits
from test_gpu_chunk import Chunks
from test_gpu_decode import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

LARGEST = 0x7F7F                          # 3.39e38


# row tiles of 128 and of 256, whole and cut, few and many pieces of a row
@pytest.mark.parametrize("hq,hkv,d,lens,news", [
    (4, 1, 64, [700, 300], [9, 300]), (4, 1, 128, [700, 3], [9, 3]), (2, 1, 64, [9000, 40], [3, 40]),
    (8, 2, 128, [20000], [700]), (8, 2, 128, [1500, 1400], [640, 640])])
@pytest.mark.parametrize("spread", [0.0, 1.0])
def test_means_of_the_largest_values(hq, hkv, d, lens, news, spread):
    s = Chunks(lens, news, hq, hkv, d, 64, seed=d, spread=spread)
    for b, (k, v) in enumerate(s.seqs):
        for t in range(len(k)):
            row = np.full((hkv, d), LARGEST, np.uint16)
            row[:, 1::2] |= 0x8000        # every other element the largest below zero
            row[:, 3] = bits(1.0)
            s.put(b, t, v=row)
    s.go()
