"""Plain float64 models of head norms, rotations and chunk attention, written from the definitions in
include/flexprefill.h and sharing no code with the library, and what bounds the kernels' errors."""
import math

import numpy as np


def frequencies(rotary, base=10000.0, scaling=None, factor=1.0, original_len=0, low_turns=1.0,
                high_turns=32.0):
    out = []
    for i in range(rotary // 2):
        if scaling == "base":
            f = (base * factor ** (rotary / (rotary - 2))) ** (-2 * i / rotary)
        else:
            f = base ** (-2 * i / rotary)
        if scaling == "linear":
            f /= factor
        if scaling == "parts":
            t = original_len * f / (2 * math.pi)
            g = min(max((t - low_turns) / (high_turns - low_turns), 0.0), 1.0)
            f = g * f + (1 - g) * f / factor
        out.append(f)
    return np.array(out)


def turn(x, positions, freq=None, layout="half", amplitude=1.0, weight=None, eps=None):
    """x [T, H, d] float64 normed (eps given) and rotated (freq given).  Returns the result and, for
    error bounds, the sum of the absolute values of what each element is the difference of."""
    y = x.copy()
    with np.errstate(all="ignore"):
        if eps is not None:
            y = y / np.sqrt((x * x).mean(2, keepdims=True) + eps)
            if weight is not None:
                y = y * weight
        if freq is None:
            return y, np.abs(y)
        n = len(freq)
        first, second = ((slice(0, n), slice(n, 2 * n)) if layout == "half"
                         else (slice(0, 2 * n, 2), slice(1, 2 * n, 2)))
        # (a turn's fraction in extended precision: a position of 2^31 times a double is off by 2^-21)
        angle = np.asarray(positions, np.longdouble)[:, None] * freq.astype(np.longdouble)
        angle = np.remainder(angle, 2 * np.arctan2(np.longdouble(0), np.longdouble(-1)))
        cos = (amplitude * np.cos(angle)).astype(np.float64)[:, None]
        sin = (amplitude * np.sin(angle)).astype(np.float64)[:, None]
        out, mass = y.copy(), np.abs(y)
        u, v = y[..., first], y[..., second]
        out[..., first], out[..., second] = u * cos - v * sin, v * cos + u * sin
        both = amplitude * (np.abs(u) + np.abs(v))
        mass[..., first], mass[..., second] = both, both
    return out, mass


def turn_tolerance(out, mass):
    """The rounding to bf16 is at most 2^-8 of the result.  Before it: cosines and sines within 2^-22
    of their size times the amplitude, the products and their difference within 3 2^-24 of the mass, a
    norm's sum of 128 squares within 128 2^-24, its root, product and weight within 2^-21: together
    below 2^-16 of the mass, here 2^-15.  Results below the smallest normal bf16 number are rounded to
    2^-134."""
    return 2.0 ** -8 * np.abs(out) + 2.0 ** -15 * mass + 2.0 ** -133


def chunk_attend(q, keys, values, scale):
    """One sequence: q [m, Hq, d], keys and values [n, Hkv, d], float64; query t sees keys 0 .. n - m +
    t.  Returns o and the sum of weight * |value|."""
    m, hq, d = q.shape
    n, hkv = keys.shape[:2]
    o, mass = np.zeros((m, hq, d)), np.zeros((m, hq, d))
    if n == 0 or m == 0:
        return o, mass
    hidden = np.arange(n) > (n - m + np.arange(m))[:, None]
    blank = hidden.all(1)
    for h in range(hq):
        g = h // (hq // hkv)
        with np.errstate(all="ignore"):
            s = q[:, h] @ keys[:, g].T * scale
            s[hidden] = -np.inf
            top = s.max(1, keepdims=True)
            w = np.exp(s - np.where(top > -np.inf, top, 0.0))
            w[hidden] = 0
            w /= np.where(blank[:, None], 1.0, w.sum(1, keepdims=True))
            odd = ~np.isfinite(values[:, g]).all(1)
            o[:, h] = w[:, ~odd] @ values[~odd, g]
            mass[:, h] = w[:, ~odd] @ np.abs(values[~odd, g])
            for j in np.nonzero(odd)[0]:         # a hidden value does not reach a row, whatever it is
                see = ~hidden[:, j]
                o[see, h] += w[see, j, None] * values[j, g]
                mass[see, h] += w[see, j, None] * np.abs(values[j, g])
    return o, mass


def chunk_tolerance(o, mass):
    """A weight is off by at most 2^-8 of itself, in O and in the sum alike: with w (1 + e) for w the
    result moves by sum w e (v - o) / sum w (1 + e), at most 2^-8 (mass + |o|) / (1 - 2^-8).  The result
    is rounded to bf16, 2^-8 |o| more.  Scores, exponentials and sums in float32: a part in 10^4 of the
    mass."""
    return 1.01 * (2.0 ** -8 * mass + 2.0 ** -7 * np.abs(o)) + 1e-4 * mass + 1e-37
