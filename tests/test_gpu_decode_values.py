"""decode_attn where values are infinite or NaN at tokens that every query sees, in own keys and in
prefixes of few and of many rows."""
import numpy as np
import pytest

from cache_model import bits
from test_gpu_decode import INF, NAN, NINF, Scene, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def put_shared(s, group, t, v):
    """Other bits for the value of token t of a group's prefix, which lies in shared pages or, past
    the last whole one, in every sequence's own."""
    for b in range(s.start[group], s.start[group + 1]):
        s.put(b, t, v=v)


def odd(s, pattern, first):
    """A value with `pattern` in every third place from `first` on."""
    v = bits(s.rng.standard_normal((s.hkv, s.d)))
    v[:, first::3] = pattern
    return v


@pytest.mark.parametrize("pattern", [INF, NINF, NAN])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (4, 2, 64), (33, 1, 64), (20, 1, 128)])
@pytest.mark.parametrize("n", [1, 40, 700])
def test_own_keys(pattern, hq, hkv, d, n):
    """At the first token, in the middle and at the last one; other columns, KV heads and
    sequences stay finite."""
    s = Scene([(0, [n, n + 9, 30])], hq, hkv, d, 16, seed=n)
    s.put(0, 0, v=odd(s, pattern, 0))
    s.put(0, n // 2, v=odd(s, pattern, 0))
    s.put(1, n + 8, v=odd(s, pattern, 1))
    s.run()


@pytest.mark.parametrize("pattern", [INF, NINF])
@pytest.mark.parametrize("count", [2, 7, 12, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_prefixes(pattern, count, d):
    """Groups of 8 to 160 rows: one or two tiles of few rows, one and two of many."""
    s = Scene([(300, [1 + 5 * (i % 7) for i in range(count)]), (77, [3, 60])], 4, 1, d, 32,
              seed=count)
    for t in (0, 131, 299):
        put_shared(s, 0, t, odd(s, pattern, 0))
    put_shared(s, 1, 40, odd(s, pattern, 2))
    s.run()


@pytest.mark.parametrize("nq", [2, 5])
def test_visible_and_late_together(nq):
    """One token that all queries see and one that only the last does, of either sign: both
    infinities in one column make NaN where both are seen."""
    s = Scene([(0, [90, 17]), (64, [20, 33])], 4, 1, 128, 16, seed=nq)
    for b in range(4):
        n = len(s.seqs[b][0])
        s.put(b, n - nq - 2, v=odd(s, INF, 0))
        s.put(b, n - 1, v=odd(s, NINF if b % 2 else INF, 0))
    s.run(nq)
