"""decode_attn on keys and values that show each range of keys by itself, so that a piece that is
lost, doubled or weighed wrongly changes a whole element of the result and not a small part of it.

Column c of the values is 1 at the tokens of some ranges and 0 elsewhere: o[c] is the weight of those
ranges, a sum without cancellation, and its error before it is rounded is relative to itself:
  - where weights are two bf16 numbers 2^-16 for them in O and as much in the sum, where they are one
    2^-8 in each; both 0 where all scores are equal, whose weights are 1;
  - 2e-5 for float32 scores, exponentials and sums.
Rounding to bf16 keeps order, so the result lies between the two bounds rounded."""
import math

import numpy as np
import pytest

from cache_model import attend, bits, floats
from test_gpu_decode import HEADS, Scene, _dev, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

WORK = 2e-5
TWO, ONE = 2 * 2.0 ** -16, 2 * 2.0 ** -8      # weights as two bf16 numbers, as one


def within(got, want, error):
    """Elements of `got` that `want`, off by up to `error`, can be rounded to."""
    low, high = floats(bits(want - error)), floats(bits(want + error))
    return (got >= low) & (got <= high)


def refill(s, keys, values):
    """keys(t, shared) and values(t, shared, b) give [len(t), d] for tokens t of sequence b;
    `shared`: the group's prefix, whose tokens are the same for all of the group."""
    for g in range(len(s.prefix)):
        for b in range(s.start[g], s.start[g + 1]):
            n = len(s.seqs[b][0])
            if n == 0:
                continue
            t = np.arange(n)
            k, v = (np.repeat(bits(f)[:, None], s.hkv, 1)
                    for f in (keys(t, s.prefix[g]), values(t, s.prefix[g], b)))
            for i, page in enumerate(s.table[s.slots[b], :-(-n // s.page)]):
                at = slice(i * s.page, min(n, (i + 1) * s.page))
                s._fill(page, 0, k[at], v[at])
            s.seqs[b] = (k, v)


def check(s, bound, nq=1, q=None):
    q = s.queries(nq) if q is None else q
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(nq))
    got = floats(o.view(torch.int16).cpu().numpy().view(np.uint16))
    for b, (k, v) in enumerate(s.seqs):
        # the KV heads hold the same, so one of them is enough for the oracle
        want, _ = attend(floats(q[b * nq:(b + 1) * nq]), floats(k[:, :1]), floats(v[:, :1]),
                         1 / math.sqrt(s.d))
        g = got[b * nq:(b + 1) * nq]
        fine = within(g, want, bound * want)
        assert fine.all(), (
            f"sequence {b}: off by {(np.abs(g - want) / np.maximum(want, 1e-30)).max():.2e} of the "
            f"element, columns {np.unique(np.nonzero(~fine)[2])[:8]}")


def tiles(d):
    """Column c: tokens of the 64-token tiles c, c + d, ..., counted from the sequence's start and
    moved by 16 so that they lie across the kernel's own."""
    return lambda t, shared, b: (((t + 16) // 64 % d)[:, None] == np.arange(d)).astype(float)


def ends(d):
    """Column c: one token alone -- around the ends of the prefix, of its steps of 16 and its tiles,
    at both ends of a sequence's own tokens, and others in between.  Tokens of the prefix have the
    first columns, the same for every sequence of the group."""
    def at(t, shared, b):
        n = len(t)
        inside = np.array([0, 1, 15, 16, 63, 64, shared // 64 * 64 - 1, shared // 64 * 64,
                           shared // 16 * 16 - 1, shared // 16 * 16, shared - 1])
        own = np.array([shared, shared + 1, shared + 15, n // 2, n - 2, n - 1])
        more = np.random.default_rng(shared).integers(0, max(shared, 1), d // 2 - len(inside))
        rest = np.random.default_rng(n).integers(shared, n, d)
        inside = np.unique(np.concatenate([inside, more]))
        own = np.unique(np.concatenate([own, rest]))
        of_all = np.concatenate([inside[(inside >= 0) & (inside < shared)],
                                 own[(own >= shared) & (own < n)]])[:d]
        x = np.zeros((n, d))
        x[of_all, np.arange(len(of_all))] = 1.0
        return x
    return at


SETS = [
    ("one of 300001", [(0, [300001])], 2, 1, 64, 256),
    ("one of 40000", [(0, [40000])], 8, 1, 128, 64),
    ("ragged", [(0, [1, 5000, 63, 64, 65, 20011, 900, 17])], 4, 2, 64, 32),
    ("few rows", [(20000, [3, 700, 64, 1])], 4, 1, 128, 64),
    ("two row tiles", [(9000, [3, 70, 1, 12, 40])], 7, 1, 128, 32),
    ("one tile of many rows", [(30011, [5 + 9 * i for i in range(12)])], 4, 1, 128, 64),
    ("clusters", [(12345, [1 + 3 * i for i in range(80)])], 4, 1, 128, 128),
    ("clusters, heads of 64", [(8000, [1 + 3 * i for i in range(50)])] * 2, 8, 2, 64, 16),
    ("groups that differ", [(5000, [3] * 70), (7003, [40] * 20), (900, [2, 600]), (0, [300])],
     4, 1, 128, 64),
]


def weights(groups, rows):
    """One bf16 number where a prefix has more than 32 rows of a KV head, two elsewhere."""
    return ONE if any(p and rows * len(own) > 32 for p, own in groups) else TWO


@pytest.mark.parametrize("name,groups,hq,hkv,d,page", SETS, ids=[x[0] for x in SETS])
@pytest.mark.parametrize("probe", [tiles, ends])
def test_equal_weights(name, groups, hq, hkv, d, page, probe):
    s = Scene(groups, hq, hkv, d, page, seed=len(name))
    refill(s, lambda t, shared: np.zeros((len(t), d)), probe(d))
    check(s, WORK)


@pytest.mark.parametrize("name,groups,hq,hkv,d,page", SETS[1:], ids=[x[0] for x in SETS[1:]])
@pytest.mark.parametrize("nq", [1, 2])
def test_weights_that_differ(name, groups, hq, hkv, d, page, nq):
    """Scores that rise and fall by 6 over the sequence, so that references move and pieces are
    joined by unequal factors."""
    if nq * sum(len(own) for _, own in groups) > 256:
        pytest.skip("as wide as with one query")
    s = Scene(groups, hq, hkv, d, page, seed=len(name) + nq)

    def keys(t, shared):
        x = np.zeros((len(t), d))
        x[:, 0] = 3.0 * np.sin(t / 700.0) + 0.37 * (t % 3)
        return x

    refill(s, keys, tiles(d))
    q = np.zeros((len(s.slots) * nq, hq, d))
    q[:, :, 0] = math.sqrt(d)            # a score is the key's first element
    check(s, WORK + weights(groups, nq * hq // hkv), nq, bits(q))


@pytest.mark.parametrize("hq,hkv,d,groups",
                         [h + ([(0, [900, 33, 4001])],) for h in HEADS]
                         + [h + ([(640, [1, 5, 64])],) for h in HEADS if 3 * h[0] // h[1] <= 32])
def test_few_rows_of_random_values(hq, hkv, d, groups):
    """Before rounding, 1e-4 of the sum of weight * |value|: two-part weights 3e-5, float32 scores of
    up to 20 and their exponentials the rest."""
    s = Scene(groups, hq, hkv, d, 32, seed=hq)
    q = s.queries(1)
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(1))
    got = floats(o.view(torch.int16).cpu().numpy().view(np.uint16))
    for b, (k, v) in enumerate(s.seqs):
        want, mass = attend(floats(q[b:b + 1]), floats(k), floats(v), 1 / math.sqrt(d))
        assert within(got[b:b + 1], want, 1e-4 * mass).all(), f"sequence {b}"
