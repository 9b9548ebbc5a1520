"""Turns of a frequency and of a position, in whole numbers of any length."""
from fractions import Fraction

_BITS = 400


def _pi():
    """pi 2^_BITS: 16 atan(1/5) - 4 atan(1/239)."""
    def atan(n):
        one = 1 << (_BITS + 20)
        power, k, total = one // n, 1, 0
        while power:
            total += power // k if k % 4 == 1 else -(power // k)
            power //= n * n
            k += 2
        return total
    return (16 * atan(5) - 4 * atan(239)) >> 20


_PI = Fraction(_pi(), 1 << _BITS)


def turns_of(f):
    """The fraction of a turn in f radians (a float or a Fraction), within 2^-300."""
    x = Fraction(f) / (2 * _PI)
    return x - x.numerator // x.denominator


def step_of(f):
    """The fraction of a turn in f radians, rounded to 2^-64."""
    return int(turns_of(f) * 2 ** 64 + Fraction(1, 2)) % 2 ** 64
