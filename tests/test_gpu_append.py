"""cache_append against the host model of the cache and float64 norms and rotations."""
import numpy as np
import pytest

from cache_model import bits, floats
from chunk_model import frequencies, turn, turn_tolerance
from test_gpu_cache import Pair, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class Append(Pair):
    """A cache and its model; keys are compared within a bound, all else bit for bit."""

    def __init__(self, hq=4, layout="half", rotary=None, norm=False, f32=False, **kw):
        super().__init__(**kw)
        d = self.dims[2]
        self.hq, self.layout = hq, layout
        rotary = d if rotary is None else rotary
        self.rope = self.fpx.Rope(rotary, layout=layout, base=5e4) if rotary else None
        self.freq = frequencies(rotary, 5e4) if rotary else None
        self.norm, self.eps, self.w = None, None, (None, None)
        if norm:
            w = 1 + 0.3 * self.rng.standard_normal((2, d))
            self.eps = 1e-5
            if f32:
                t = torch.from_numpy(w.astype(np.float32)).cuda()
                self.w = tuple(w.astype(np.float32).astype(np.float64))
            else:
                t = self._dev(bits(w))
                self.w = tuple(floats(bits(w)))
            self.norm = self.fpx.HeadNorm(t[0], t[1], self.eps)
        self.want = {}                       # (layer, page, head, row): key row and its mass

    def put(self, slots, counts, in_place=False, queries=True):
        layers, hkv, d = self.dims
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        T = int(cu[-1])
        place = np.concatenate([np.arange(c) + self.m.len[s] - c for s, c in zip(slots, counts)]
                               + [np.zeros(0, int)])
        for layer in range(layers):
            x = bits(1.5 * self.rng.standard_normal((T, self.hq + 2 * hkv, d)))
            k, v = x[:, self.hq:self.hq + hkv], x[:, self.hq + hkv:]
            kt, mass = turn(floats(k), place, self.freq, self.layout, 1.0, self.w[1], self.eps)
            self.m.write(layer, bits(kt), v, slots, cu)
            for i, s in enumerate(slots):
                for j in range(cu[i], cu[i + 1]):
                    t = place[j]
                    if t >= 0:
                        p = self.m.rows[s][t // self.m.page]
                        self.want[layer, p, t % self.m.page] = kt[j], mass[j]
            t = self._dev(x)
            out = t[:, :self.hq] if in_place else None
            q = self.fpx.cache_append(self.c, layer, t[:, :self.hq] if queries else None,
                                      t[:, self.hq:self.hq + hkv], t[:, self.hq + hkv:], slots, cu,
                                      self.rope, self.norm, q_out=out)
            if not queries:
                assert q is None
                continue
            want, mass = turn(floats(x[:, :self.hq]), place, self.freq, self.layout, 1.0, self.w[0],
                              self.eps)
            there = place >= 0
            err = np.abs(floats(_bits(q)) - want)[there]
            assert np.all(err <= turn_tolerance(want, mass)[there])
            if in_place:
                assert q.data_ptr() == t.data_ptr()
            assert np.array_equal(_bits(t)[:, self.hq:], x[:, self.hq:])

    def same(self):
        self.c.check()
        assert np.array_equal(self.c.meta.cpu().numpy(), self.m.meta())
        assert np.array_equal(_bits(self.c.v), self.m.v)
        got, rest = _bits(self.c.k), self.m.k.copy()
        for (layer, p, r), (kt, mass) in self.want.items():
            err = np.abs(floats(got[layer, p, :, r]) - kt)
            assert np.all(err <= turn_tolerance(kt, mass)), (layer, p, r)
            rest[layer, p, :, r] = got[layer, p, :, r]
        assert np.array_equal(got, rest)          # nothing else was written


@pytest.mark.parametrize("d,hkv,hq", [(64, 2, 4), (128, 1, 7), (128, 3, 48), (64, 16, 17)])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("layout,norm", [("half", False), ("half", True), ("interleaved", True)])
def test_growing_sequences(d, hkv, hq, page, layout, norm):
    a = Append(hq, layout, norm=norm, layers=1, pages=64, hkv=hkv, d=d, slots=5, max_pages=20, page=page,
               seed=d + hq + page)
    for slots, counts in (([3, 0, 1], [1, 70, 15]), ([1, 3], [1, 1]), ([0, 1, 3, 4], [64, 17, 0, 129]),
                          ([4, 0], [1, 63])):
        a.reserve(slots, counts)
        a.put(slots, counts)
    a.same()


@pytest.mark.parametrize("rotary", [0, 16, 48])
@pytest.mark.parametrize("norm,f32", [(False, False), (True, True)])
@pytest.mark.parametrize("queries,in_place", [(True, True), (False, False)])
def test_parts_weights_and_queries(rotary, norm, f32, queries, in_place):
    a = Append(6, "half", rotary, norm, f32, layers=2, pages=30, hkv=2, d=64, slots=3, max_pages=10,
               page=32, seed=rotary)
    a.reserve([2, 0], [100, 3])
    a.put([2, 0], [100, 3], in_place, queries)
    a.reserve([0, 2], [30, 1])
    a.put([0, 2], [30, 1], in_place, queries)
    a.same()


def test_equal_to_rotate_and_write():
    """Bit for bit what rotate and cache_write leave."""
    import paper_2502_20766_amd as fpx
    g = torch.Generator("cuda").manual_seed(1)
    n, hq, hkv, d = 333, 8, 2, 128
    x = torch.randn(n, hq + 2 * hkv, d, generator=g, device="cuda").bfloat16()
    w = torch.randn(2, d, generator=g, device="cuda").bfloat16()
    rope, norm = fpx.Rope(d, base=1e6), fpx.HeadNorm(w[0], w[1])
    one, two = (fpx.Cache(1, 12, hkv, d, 2, 8, 64) for _ in range(2))
    for c in (one, two):
        c.k.zero_(), c.v.zero_()
        fpx.cache_reserve(c, [1], n)
    q = fpx.cache_append(one, 0, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], [1], [0, n], rope, norm)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    q2, k2 = fpx.rotate(x[:, :hq], x[:, hq:hq + hkv], pos, rope, norm)
    fpx.cache_write(two, 0, k2, x[:, hq + hkv:], [1], [0, n])
    assert torch.equal(q, q2) and torch.equal(one.k, two.k) and torch.equal(one.v, two.v)


def test_more_rows_than_tokens():
    """Rows beyond a slot's length are left out, and their rows of q_out stay."""
    a = Append(4, layers=1, pages=10, hkv=2, d=64, slots=2, max_pages=6, page=16)
    a.reserve([1], [5])
    x = a._dev(bits(a.rng.standard_normal((9, 8, 64))))
    out = torch.full((9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    a.fpx.cache_append(a.c, 0, x[:, :4], x[:, 4:6], x[:, 6:], [1], [0, 9], a.rope, q_out=out)
    want, _ = a.fpx.rotate(x[4:, :4], None, torch.arange(5, dtype=torch.int32, device="cuda"), a.rope)
    assert torch.equal(out[4:], want) and bool((out[:4] == 7).all())
    a.c.check()


def test_nothing_after_a_failed_reserve():
    a = Append(4, layers=1, pages=4, hkv=2, d=64, slots=3, max_pages=4, page=16)
    a.append([0], [20])
    a.reserve([1], [100])                     # too few pages
    before = _bits(a.c.k), _bits(a.c.v)
    x = a._dev(bits(a.rng.standard_normal((5, 8, 64))))
    out = torch.full((5, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    a.fpx.cache_append(a.c, 0, x[:, :4], x[:, 4:6], x[:, 6:], [0], [0, 5], a.rope, q_out=out)
    assert np.array_equal(before[0], _bits(a.c.k)) and np.array_equal(before[1], _bits(a.c.v))
    assert bool((out == 7).all())
    with pytest.raises(a.fpx.CacheError):
        a.c.check()
    a.fpx.cache_append(a.c, 0, x[:, :4], x[:, 4:6], x[:, 6:], [0], [0, 5], a.rope, q_out=out)
    a.c.check()
    assert not bool((out == 7).all(2).any())


def test_shared_pages_are_left_alone():
    a = Append(4, layers=1, pages=8, hkv=1, d=64, slots=3, max_pages=4, page=16)
    a.append([0], [20])
    a.fork([0], [2])
    before = _bits(a.c.k), _bits(a.c.v)
    x = a._dev(bits(a.rng.standard_normal((2, 6, 64))))
    a.fpx.cache_append(a.c, 0, x[:, :4], x[:, 4:5], x[:, 5:], [2], [0, 2], a.rope)   # not reserved
    assert np.array_equal(before[0], _bits(a.c.k)) and np.array_equal(before[1], _bits(a.c.v))
    with pytest.raises(a.fpx.CacheError) as e:
        a.c.check()
    assert e.value.bits == a.fpx.CACHE_SHARED


def test_a_slot_that_is_full_to_its_last_place():
    a = Append(2, norm=True, layers=1, pages=9, hkv=1, d=128, slots=2, max_pages=4, page=16)
    a.reserve([1], [64])
    a.put([1], [64])
    a.same()


def test_refusals():
    import paper_2502_20766_amd as fpx
    c = fpx.Cache(1, 4, 2, 64, 2, 4, 16)
    x = torch.zeros(3, 8, 64, dtype=torch.bfloat16, device="cuda")
    q, k, v, rope = x[:, :4], x[:, 4:6], x[:, 6:], fpx.Rope(64)
    for call in (lambda: fpx.cache_append(c, 0, q.float(), k, v, [0], [0, 3], rope),
                 lambda: fpx.cache_append(c, 0, q[:2], k, v, [0], [0, 3], rope),
                 lambda: fpx.cache_append(c, 0, q, k, v, [0], [0, 2], rope),
                 lambda: fpx.cache_append(c, 0, q, k, v, [0, 1], [0, 3], rope),
                 lambda: fpx.cache_append(c, 0, q, q, v, [0], [0, 3], rope),
                 lambda: fpx.cache_append(c, 0, q, k, v, [0], [0, 3], rope, q_out=k),
                 lambda: fpx.cache_append(c, 0, None, k, v, [0], [0, 3], rope, q_out=q),
                 lambda: fpx.cache_append(c, 0, q.cpu(), k, v, [0], [0, 3], rope),
                 lambda: fpx.cache_append(c, 0, q, k, v, [0], [0, 3], rope,
                                          fpx.HeadNorm(torch.ones(128, device="cuda")))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fpx.FlexPrefillError):
        fpx.cache_append(c, 0, q, k, v, [0], [0, 3], fpx.Rope(128))
    with pytest.raises(fpx.FlexPrefillError):
        fpx.cache_append(c, 1, q, k, v, [0], [0, 3], rope)


@pytest.mark.parametrize("d,hkv,hq", [(64, 1, 1), (64, 1, 2), (128, 1, 3), (128, 2, 4), (64, 1, 5),
                                      (64, 3, 6), (64, 1, 15), (128, 1, 8)])
@pytest.mark.parametrize("norm", [False, True])
def test_few_query_heads(d, hkv, hq, norm):
    """Queries of several tokens side by side; parts of the 64 positions of 8 to 64 tokens."""
    a = Append(hq, norm=norm, layers=1, pages=64, hkv=hkv, d=d, slots=5, max_pages=20, page=16, seed=d + hq)
    for slots, counts in (([3, 0, 1], [1, 70, 15]), ([1, 3], [1, 1]), ([0, 1, 3, 4], [64, 17, 0, 129]),
                          ([4, 0], [1, 63])):
        a.reserve(slots, counts)
        a.put(slots, counts)
    a.same()
