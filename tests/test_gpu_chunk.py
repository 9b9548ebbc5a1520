"""chunk_attn against float64 on the host, element by element."""
import math

import numpy as np
import pytest

from cache_model import bits, floats
from chunk_model import chunk_attend, chunk_tolerance
from test_gpu_decode import Scene, _dev, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Chunks(Scene):
    """Sequences of `lens` tokens (None: no slot) with `news` queries each."""

    def __init__(self, lens, news, hq, hkv, d, page=64, seed=0, **kw):
        super().__init__([(0, list(lens))], hq, hkv, d, page, seed, **kw)
        self.news = list(news)
        self.cu = np.concatenate([[0], np.cumsum(self.news)]).astype(np.int32)

    def q_bits(self, scale=1.5):
        return bits(self.rng.standard_normal((int(self.cu[-1]), self.hq, self.d)) * scale)

    def of(self, softmax_scale=0.0):
        return self.fpx.ChunkBatch(self.slots, self.cu, self.hq, softmax_scale)

    def verify(self, q, o, scale=None):
        scale = scale or 1 / math.sqrt(self.d)
        got = floats(_bits(o))
        for b, (k, v) in enumerate(self.seqs):
            at = slice(self.cu[b], self.cu[b + 1])
            want, mass = chunk_attend(floats(q[at]), floats(k), floats(v), scale)
            g = got[at]
            fine = np.isfinite(want)
            assert np.array_equal(fine, np.isfinite(g)), f"sequence {b}: other finite places"
            assert np.array_equal(want[~fine & ~np.isnan(want)], g[~fine & ~np.isnan(want)])
            err, tol = np.abs(g - want)[fine], chunk_tolerance(want, mass)[fine]
            assert np.all(err <= tol), (f"sequence {b}: {err.max():.3e}, "
                                        f"{(err / tol).max():.2f} of the bound")

    def go(self, softmax_scale=0.0, qscale=1.5, q=None):
        q = self.q_bits(qscale) if q is None else q
        o = self.fpx.chunk_attn(_dev(q), self.cache(), 0, self.of(softmax_scale))
        self.verify(q, o, softmax_scale or None)
        return q, o


HEADS = [(4, 1, 128), (2, 2, 64), (16, 1, 64), (7, 1, 128), (8, 2, 64), (1, 1, 128), (33, 1, 64),
         (130, 1, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("n,m", [(1, 1), (2, 1), (16, 16), (17, 5), (63, 63), (64, 64), (65, 65), (65, 1),
                                 (128, 64), (129, 127), (200, 33), (1000, 31), (1000, 1), (300, 300)])
def test_one_sequence(hq, hkv, d, n, m):
    Chunks([n], [m], hq, hkv, d, seed=n + m).go()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (8, 2, 64), (7, 1, 64)])
def test_ragged_batch(page, hq, hkv, d):
    """Lengths around every boundary, empty and idle slots, sequences without queries, more queries
    than tokens."""
    lens = [1, 700, 16, None, 63, 64, 65, 0, 3, 257, 128, 15, 17, 400, None, 90]
    news = [1, 300, 16, 3, 20, 0, 64, 5, 9, 1, 128, 15, 2, 399, 40, 0]
    Chunks(lens, news, hq, hkv, d, page, seed=page).go()


@pytest.mark.parametrize("count", [60, 256])
def test_many_sequences(count):
    """Up to the largest batch; most with one query."""
    lens = [1 + (37 * i) % 150 for i in range(count)]
    news = [1 + (i % 17 == 3) * (i % 40) for i in range(count)]
    Chunks(lens, news, 4, 1, 64, 16, seed=count).go()
    Chunks(lens, news, 4, 2, 128, 16, seed=count).go()


@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (2, 1, 64)])
@pytest.mark.parametrize("n,m", [(9000, 700), (20011, 3), (6000, 1500)])
def test_long_sequences(hq, hkv, d, n, m):
    Chunks([n], [m], hq, hkv, d, 64, seed=m).go()


def test_long_and_short_sequences_together():
    lens = [9000, 5, 300, 4097, 64, 700, 2]
    news = [257, 5, 1, 64, 1, 700, 1]
    Chunks(lens, news, 8, 2, 128, 32, seed=9).go()
    Chunks(lens, news, 4, 4, 64, 128, seed=9).go()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,news", [([777], [777]), ([5000], [130]), ([3000, 40, 900], [1, 40, 333])])
def test_every_key_counts_once(d, lens, news):
    """Queries of zero weigh all keys alike: each result is the mean of the values that a row sees,
    whole numbers that float32 sums exactly, so only the mean's division and rounding err.  Every
    value differs from its neighbours, and one key in the middle holds a large one."""
    s = Chunks(lens, news, 4, 2, d, 16, seed=d)
    for b, (k, v) in enumerate(s.seqs):
        for t in range(len(k)):
            s.put(b, t, v=bits(np.full((2, d), (t * 7) % 31 - 15.0) + (np.arange(d) % 3)))
        s.put(b, len(k) // 2, v=bits(np.full((2, d), 256.0)))
    q = np.zeros((int(s.cu[-1]), 4, d), np.uint16)
    o = floats(_bits(s.fpx.chunk_attn(_dev(q), s.cache(), 0, s.of())))
    for b, (k, v) in enumerate(s.seqs):
        n, m = len(k), s.news[b]
        total = np.cumsum(floats(v), 0)[n - m:] / np.arange(n - m + 1, n + 1)[:, None, None]
        got, want = o[s.cu[b]:s.cu[b + 1]], np.repeat(total, 2, 1)
        # 2^-8 for the rounding, 2^-20 for the reciprocal and product (and the merge of ranges)
        assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(want) + 1e-6)


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan, 3.3e38])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (2, 2, 64)])
def test_values_that_later_rows_see(value, hq, hkv, d):
    """A key or a value that is not finite reaches the rows that see it and no other."""
    for t, where in ((150, "v"), (150, "k"), (199, "v"), (64, "v"), (99, "kv"), (0, "v")):
        s = Chunks([200, 70], [120, 70], hq, hkv, d, 32, seed=t)
        row = s.seqs[0][0 if where == "k" else 1][t].copy()
        row[0, 5] = bits(value)
        if "k" in where:
            key = s.seqs[0][0][t].copy()
            key[0, 3] = bits(np.nan if value == 3.3e38 else value)
            s.put(0, t, k=key)
        if "v" in where:
            s.put(0, t, v=row)
        q = s.q_bits()
        if "k" in where and np.isinf(value):   # the sign of the score decides: +inf - inf is NaN
            q[..., 3] &= 0x7FFF
            if value > 0:
                o = floats(_bits(s.fpx.chunk_attn(_dev(q), s.cache(), 0, s.of())))
                g = hq // hkv
                sees = np.arange(80, 200) >= t
                assert np.isnan(o[:120][sees][:, :g]).all()
                assert np.isfinite(o[:120][~sees]).all() and np.isfinite(o[120:]).all()
                continue
        s.go(q=q)


@pytest.mark.parametrize("d", [64, 128])
def test_several_values_that_are_not_finite(d):
    s = Chunks([130, 66], [130, 2], 4, 2, d, 16, seed=d)
    for b, t, h, e, x in ((0, 10, 0, 3, np.inf), (0, 10, 1, 9, -np.inf), (0, 64, 0, 3, np.inf),
                          (0, 100, 0, 40, np.nan), (0, 129, 1, 9, np.inf), (1, 65, 0, 0, np.inf)):
        row = s.seqs[b][1][t].copy()
        row[h, e] = bits(x)
        s.put(b, t, v=row)
    s.go()


def test_scores_that_rise_and_weights_that_vanish():
    """References that move often, scores far apart, a scale of the caller."""
    s = Chunks([3000, 500], [90, 500], 4, 2, 128, 64, seed=2, spread=4.0)
    s.go(qscale=4.0)
    s.go(softmax_scale=0.7)
    s.go(softmax_scale=1e-6)
    for t in range(0, 3000, 50):                 # keys ever further along the queries
        s.put(0, t, k=bits(np.full((2, 128), 0.002 * t)))
    s.go(q=bits(np.abs(s.rng.standard_normal((590, 4, 128)))))


def test_strided_queries_and_what_lies_around():
    s = Chunks([500, 40], [33, 40], 4, 2, 128, 64, seed=4)
    q = s.q_bits()
    wide = np.full((73, 7, 128), 0x7FC1, np.uint16)
    wide[:, 2:6] = q
    out = torch.full((75, 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    c, b = s.cache(), s.of()
    n = s.fpx.chunk_workspace_size(c, b)
    ws = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    s.fpx.chunk_attn(_dev(wide)[:, 2:6], c, 0, b, out=out[1:74], workspace=ws[:n])
    s.verify(q, out[1:74])
    assert bool((out[0] == 5).all()) and bool((out[74] == 5).all()) and bool((ws[n:] == 0x5A).all())


def test_the_same_call_gives_the_same_bits():
    s = Chunks([9000, 70, 4000], [200, 70, 1], 8, 2, 128, 64, seed=5)
    q, c, b = _dev(s.q_bits()), s.cache(), s.of()
    one = s.fpx.chunk_attn(q, c, 0, b)
    ws = torch.full((s.fpx.chunk_workspace_size(c, b),), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(5):
        assert torch.equal(one, s.fpx.chunk_attn(q, c, 0, b, workspace=ws))


def test_a_slot_twice_and_the_other_layers():
    """Two chunks over one slot; layers apart from each other."""
    import paper_2502_20766_amd as fpx
    g = torch.Generator("cuda").manual_seed(0)
    c = fpx.Cache(3, 20, 2, 64, 3, 10, 16)
    n = 150
    kv = torch.randn(3, 2, n, 2, 64, generator=g, device="cuda").bfloat16()
    fpx.cache_reserve(c, [1], n)
    for layer in range(3):
        fpx.cache_write(c, layer, kv[layer, 0], kv[layer, 1], [1], [0, n])
    q = torch.randn(70, 4, 64, generator=g, device="cuda").bfloat16()
    for layer in range(3):
        o = floats(_bits(fpx.chunk_attn(q, c, layer, fpx.ChunkBatch([1, 1], [0, 20, 70], 4))))
        k, v = (x.double().cpu().numpy() for x in kv[layer])
        for a, b in ((0, 20), (20, 70)):
            want, mass = chunk_attend(q[a:b].double().cpu().numpy(), k, v, 0.125)
            assert np.all(np.abs(o[a:b] - want) <= chunk_tolerance(want, mass))


def test_a_table_that_names_no_page():
    """Entries outside the pool (a caller's own bookkeeping) read some page of it, never past it."""
    s = Chunks([300], [40], 4, 1, 64, 16, seed=6)
    s.k[:], s.v[:] = bits(0.5), bits(0.25)       # whatever page is read
    c = s.cache()
    c.table[int(s.slots[0]), 3:7] = torch.tensor([-1, 2 ** 30, -2 ** 31, s.total], dtype=torch.int32)
    o = s.fpx.chunk_attn(_dev(s.q_bits()), c, 0, s.of())
    assert bool((o == 0.25).all())


def test_refusals():
    import paper_2502_20766_amd as fpx
    c = fpx.Cache(1, 4, 2, 64, 2, 4, 16)
    b = fpx.ChunkBatch([0], [0, 3], 4)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(fpx.chunk_workspace_size(c, b), dtype=torch.uint8, device="cuda")
    for call in (lambda: fpx.chunk_attn(q[:2], c, 0, b), lambda: fpx.chunk_attn(q.half(), c, 0, b),
                 lambda: fpx.chunk_attn(q[:, :2], c, 0, b), lambda: fpx.chunk_attn(q.cpu(), c, 0, b),
                 lambda: fpx.chunk_attn(q, c, 0, b, out=q[:2]),
                 lambda: fpx.chunk_attn(q, c, 0, b, workspace=ws.view(torch.int32)),
                 lambda: fpx.chunk_attn(q.transpose(0, 1), c, 0, b)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fpx.FlexPrefillError):
        fpx.chunk_attn(q, c, 0, b, workspace=ws[:-1])
    with pytest.raises(fpx.FlexPrefillError):
        fpx.chunk_attn(q, c, 1, b)


@pytest.mark.parametrize("hq,hkv,d,m", [(4, 1, 64, 3), (4, 1, 128, 3), (4, 2, 128, 300)])
@pytest.mark.parametrize("n", [1200, 30000])
def test_values_that_are_not_finite_behind_vanishing_weights(hq, hkv, d, m, n):
    """A weight that float32 rounds to zero times infinity is not finite, also where the keys of such
    weights make up whole pieces of a sequence that is cut."""
    s = Chunks([n], [m], hq, hkv, d, 64, seed=n)
    low, zero = bits(np.full((hkv, d), -256.0)), bits(np.zeros((hkv, d)))
    for t in range(n):
        s.put(0, t, k=low if t < n // 2 else zero)
    row = s.seqs[0][1][10].copy()
    row[0, 5] = bits(np.inf)
    s.put(0, 10, v=row)
    q = bits(np.ones((m, hq, d)))
    o = floats(_bits(s.fpx.chunk_attn(_dev(q), s.cache(), 0, s.of())))
    odd = np.zeros((hq, d), bool)
    odd[:hq // hkv, 5] = True
    assert not np.isfinite(o[:, odd]).any() and np.isfinite(o[:, ~odd]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("n", [880, 895, 896, 897, 911, 960, 961])
def test_where_sequences_begin_to_be_cut(d, page, n):
    """Lengths about 14 key tiles, to which sequences stay whole whatever the rest, one launch if the
    table has room for no more; alone, and beside short and idle ones."""
    Chunks([n], [1], 4, 1, d, page, seed=n).go()
    Chunks([n, 3, None, 400, 0, n - 1], [200, 3, 2, 1, 4, 33], 4, 2, d, page, seed=n).go()


@pytest.mark.parametrize("d", [64, 128])
def test_whole_row_tiles_of_many_sequences(d):
    """More row tiles than workgroups at a time, of which none is cut, and the same with one sequence so
    long that they are."""
    lens, news = [700 + 13 * i for i in range(40)], [120 + 11 * i for i in range(40)]
    Chunks(lens, news, 4, 4, d, 64, seed=d).go()
    Chunks(lens + [20000], news + [2], 4, 4, d, 64, seed=d).go()


def test_whole_row_tiles_of_256():
    """Prompts that fill row tiles of 256, of which none is cut; a row tile that ends a sequence early."""
    Chunks([1025, 900, 1100, None, 960, 0], [1025, 900, 1100, 5, 960, 3], 8, 2, 128, 64, seed=1).go()
    Chunks([1500, 1400, 1300], [640, 640, 576], 8, 4, 128, 32, seed=2).go()
