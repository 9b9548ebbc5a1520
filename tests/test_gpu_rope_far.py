"""Cosines and sines of rotate at far positions and large frequencies, element by element, against angles
in whole numbers of any length."""
import math

import numpy as np
import pytest

from cache_model import floats
from rope_turns import turns_of
from test_gpu_rope import _bits, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

SETS = {
    "large": [8191.7, -8191.7, 1e5, 99999.99, 1048575.3, 2.0 ** 20, -1048575.3, 524287.77],
    "usual": [500000.0 ** (-i / 8) for i in range(8)],
    "small": [2.0 ** -20, 1e-9, 2.0 ** -31, -2.0 ** -31, 1e-12, 0.0, 2.0 ** -63, 5e-324],
}


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_cosines_and_sines(gpu, name, layout):  # noqa: F811
    """Heads whose pairs are (1, 0) become (cos, sin): within 2^-22, and the rounding to bf16, 2^-8 of
    the result."""
    rng = np.random.default_rng(0)
    top = 2 ** 31
    pos = np.concatenate([[0, 1, -1, top - 1, -top, 1 - top], rng.integers(-top, top, 500),
                          rng.integers(0, 200000, 300)])
    f = SETS[name]
    x = torch.zeros(len(pos), 1, 64, dtype=torch.bfloat16, device="cuda")
    first, second = (slice(0, 8), slice(8, 16)) if layout == "half" else (slice(0, 16, 2), slice(1, 16, 2))
    x[..., first] = 1
    out, _ = gpu.rotate(x, None, torch.from_numpy(pos.astype(np.int32)).cuda(),
                        gpu.Rope(16, layout=layout, inv_freq=f))
    got = floats(_bits(out))[:, 0]
    turn = [turns_of(v) for v in f]
    angle = np.array([[2 * math.pi * float(int(p) * t % 1) for t in turn] for p in pos])
    for part, want in ((got[:, first], np.cos(angle)), (got[:, second], np.sin(angle))):
        err, tol = np.abs(part - want), 2.0 ** -8 * (np.abs(want) + 2.0 ** -22) + 2.0 ** -22
        assert np.all(err <= tol), f"{(err / tol).max():.2f} of the bound"
