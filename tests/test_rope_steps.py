"""The fractions of a turn that fp_rope_init makes of frequencies, against whole-number arithmetic of any
length (these run without a GPU)."""
import math

import numpy as np
import pytest

import paper_2502_20766_amd as fpx
from rope_turns import step_of
from test_rope_abi import lib  # noqa: F401

FREQUENCIES = [1.0, 0.1, 3.7, -0.25, 1023.9, 8191.7, -8191.7, 1e5, 99999.99, -1e5, 1048575.3, 2.0 ** 20,
               -(2.0 ** 20), math.nextafter(2.0 ** 20, 0), 2 * math.pi, math.pi * 1e5, 2.0 ** -30,
               2.0 ** -63, 2.0 ** -64, 2.0 ** -80, 5e-324, -5e-324, 0.0, -0.0]


def steps(f):
    f = list(f) + [0.0] * (-len(f) % 64)
    return [int(x) for i in range(0, len(f), 64)
            for x in fpx.Rope(128, inv_freq=f[i:i + 64]).c.step]


def off(got, f):
    """Units of 2^-64 of a turn."""
    want = step_of(f)
    return min((got - want) % 2 ** 64, (want - got) % 2 ** 64)


def test_the_model_itself():
    """Fractions that are known: pi to 30 digits gives the turns of a radian."""
    pi = 314159265358979323846264338328
    assert abs(step_of(1.0) - 2 ** 64 * 10 ** 29 // (2 * pi)) <= 1
    assert step_of(0.0) == 0 and (step_of(-3.5) + step_of(3.5)) % 2 ** 64 == 0


def test_frequencies_to_the_last_bit(lib):  # noqa: F811
    """Rounded to 2^-64 of a turn, so that a position of 2^31 is off by 2^-33 of one, for whole turns as
    well as for none."""
    for f, got in zip(FREQUENCIES, steps(FREQUENCIES)):
        assert off(got, f) <= 1, f


@pytest.mark.parametrize("seed", range(4))
def test_drawn_frequencies(lib, seed):  # noqa: F811
    rng = np.random.default_rng(seed)
    f = 2.0 ** rng.uniform(-70, 20, 2000) * rng.choice([-1, 1], 2000)
    for x, got in zip(f, steps(f)):
        assert off(got, float(x)) <= 1, x


def test_frequencies_of_a_base(lib):  # noqa: F811
    """Powers of a base, as float64 numbers."""
    for base in (1e4, 5e5, 1.0, 0.01):
        for i, got in enumerate(fpx.Rope(128, base=base).c.step):
            assert off(int(got), math.pow(base, -2.0 * i / 128)) <= 1
