"""decode_attn against float64 on the host, element by element, with an error bound that is
little more than the rounding of the result to bf16 (cache_model.tolerance)."""
import math

import numpy as np
import pytest

from cache_model import attend, bits, floats, tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_20766_amd as fpx
    fpx.lib()
    return fpx


def _dev(x):
    return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)


class Scene:
    """Groups of sequences that share prefixes, in a cache whose pages are shuffled and whose
    free places hold NaN; the tokens also on the host."""

    def __init__(self, groups, hq, hkv, d, page=64, seed=0, spread=1.0, gain=1.0):
        # groups: [(prefix tokens, [own tokens of each sequence, None: idle])]
        import paper_2502_20766_amd as fpx
        self.fpx, self.rng = fpx, np.random.default_rng(seed)
        self.hq, self.hkv, self.d, self.page = hq, hkv, d, page
        rng = self.rng
        seqs = [(g, n) for g, (_, own) in enumerate(groups) for n in own]
        batch = len(seqs)
        total = sum(-(-(p + (n or 0)) // page) for (p, own) in groups for n in own) + 4
        rows = max(1, max(-(-(groups[g][0] + (n or 0)) // page) for g, n in seqs))
        nan = lambda shape: np.full(shape, 0x7FC1, np.uint16)     # noqa: E731
        self.k = nan((1, total, hkv, page, d))
        self.v = nan((1, total, hkv, page // 16, d, 16))
        slots = rng.permutation(batch + 2)[:batch]
        self.slots = np.where([n is None for _, n in seqs], -1, slots).astype(np.int32)
        lens = np.zeros(batch + 2, np.int32)
        table = np.full((batch + 2, rows), -1, np.int32)
        free = list(rng.permutation(total))
        commons = []
        for p, own in groups:
            kp = bits(rng.standard_normal((p, hkv, d)) * spread)
            vp = bits(rng.standard_normal((p, hkv, d)) * gain)
            pages = [free.pop() for _ in range(p // page)]
            for i, pg in enumerate(pages):
                self._fill(pg, 0, kp[i * page:(i + 1) * page], vp[i * page:(i + 1) * page])
            commons.append((kp, vp, pages))
        self.seqs = []
        for b, (g, n) in enumerate(seqs):
            if n is None:
                self.seqs.append((np.zeros((0, hkv, d), np.uint16),) * 2)
                continue
            kp, vp, pages = commons[g]
            k = np.concatenate([kp, bits(rng.standard_normal((n, hkv, d)) * spread)])
            v = np.concatenate([vp, bits(rng.standard_normal((n, hkv, d)) * gain)])
            row = list(pages)
            for at in range(len(pages) * page, len(k), page):
                pg = free.pop()
                self._fill(pg, 0, k[at:at + page], v[at:at + page])
                row.append(pg)
            lens[slots[b]] = len(k)
            table[slots[b], :len(row)] = row
            self.seqs.append((k, v))
        meta = np.zeros(8 + 2 * -(-total // 64) + batch + 2 + total, np.int32)
        meta[8 + 2 * -(-total // 64):][:batch + 2] = lens
        self.meta = np.concatenate([meta, table.ravel()])
        self.lens_at = 8 + 2 * -(-total // 64)
        self.table, self.lens, self.total, self.rows = table, lens, total, rows
        self.start = np.concatenate([[0], np.cumsum([len(own) for _, own in groups])])
        self.prefix = [p for p, _ in groups]

    def _fill(self, page, at, k, v):
        for h in range(self.hkv):
            self.k[0, page, h, at:at + len(k)] = k[:, h]
            for r in range(0, len(v), 16):
                self.v[0, page, h, r // 16, :, :len(v[r:r + 16])] = v[r:r + 16, h].T

    def put(self, b, t, k=None, v=None):
        """Other bits for token t of sequence b (not one that others share)."""
        pg = self.table[self.slots[b], t // self.page]
        r = t % self.page
        if k is not None:
            self.k[0, pg, :, r], self.seqs[b][0][t] = k, k
        if v is not None:
            self.v[0, pg, :, r // 16, :, r % 16], self.seqs[b][1][t] = v, v

    def cache(self):
        return self.fpx.Cache(1, self.total, self.hkv, self.d, len(self.lens), self.rows,
                              self.page, k=_dev(self.k), v=_dev(self.v),
                              meta=torch.from_numpy(self.meta).cuda())

    def queries(self, nq, scale=1.5):
        return bits(self.rng.standard_normal((len(self.slots) * nq, self.hq, self.d)) * scale)

    def batch(self, nq, shared=True, softmax_scale=0.0):
        if not shared:
            return self.fpx.DecodeBatch(self.slots, self.hq, nq, softmax_scale=softmax_scale)
        return self.fpx.DecodeBatch(self.slots, self.hq, nq, self.start, self.prefix,
                                    softmax_scale)

    def check(self, q, o, nq, scale=None):
        scale = scale or 1 / math.sqrt(self.d)
        got = floats(o.view(torch.int16).cpu().numpy().view(np.uint16))
        for b, (k, v) in enumerate(self.seqs):
            want, mass = attend(floats(q[b * nq:(b + 1) * nq]), floats(k), floats(v), scale)
            g = got[b * nq:(b + 1) * nq]
            fine = np.isfinite(want)
            assert np.array_equal(fine, np.isfinite(g)), f"sequence {b}: other finite places"
            assert np.array_equal(want[~fine & ~np.isnan(want)], g[~fine & ~np.isnan(want)])
            err = np.abs(g[fine] - want[fine])
            tol = tolerance(want, mass)[fine]
            assert np.all(err <= tol), (f"sequence {b}: {err.max():.3e}, "
                                        f"{(err / tol).max():.2f} of the bound")

    def run(self, nq=1, shared=True, softmax_scale=0.0, qscale=1.5):
        q = self.queries(nq, qscale)
        o = self.fpx.decode_attn(_dev(q), self.cache(), 0, self.batch(nq, shared, softmax_scale))
        self.check(q, o, nq, softmax_scale or None)
        return q, o


HEADS = [(4, 1, 128), (2, 2, 64), (16, 1, 64), (7, 1, 128), (8, 2, 64), (48, 1, 128),
         (17, 1, 64), (33, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 1000])
def test_one_sequence(hq, hkv, d, n):
    Scene([(0, [n])], hq, hkv, d, seed=n).run()


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("nq", [1, 2, 5, 16])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (8, 2, 64)])
def test_ragged_batch(page, nq, hq, hkv, d):
    """Lengths around every boundary, empty and idle slots, more queries than tokens."""
    own = [1, 700, 16, None, 63, 64, 65, 0, 3, 257, 128, 15, 17]
    Scene([(0, own)], hq, hkv, d, page, seed=page + nq).run(nq, shared=False)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 64, 100, 640, 1500])
def test_shared_prefix(hq, hkv, d, prefix):
    Scene([(prefix, [1, 5, 64, 90])], hq, hkv, d, 32, seed=prefix).run()


@pytest.mark.parametrize("nq", [1, 3, 16])
@pytest.mark.parametrize("count", [2, 9, 33, 70])
def test_rows_of_a_group(nq, count):
    """Row tiles of 128: from a few rows to several tiles, the last not full."""
    own = [16 + (7 * i) % 50 for i in range(count)]
    Scene([(333, own)], 4, 1, 128, 64, seed=count + nq).run(nq)
    Scene([(333, own)], 4, 2, 64, 64, seed=count + nq).run(nq)


@pytest.mark.parametrize("sizes", [(40, 40), (40, 100), (33, 33, 33), (90, 2, 90), (65, 7, 1, 33)])
@pytest.mark.parametrize("prefix", [70, 900])
def test_row_tiles_of_several_groups(sizes, prefix):
    """Groups with as many row tiles as each other (taken side by side) and with others, beside
    groups of few rows and sequences of their own."""
    groups = [(prefix + 50 * i, [1 + (11 * j) % 40 for j in range(n)])
              for i, n in enumerate(sizes)]
    Scene(groups, 4, 1, 128, 32, seed=sum(sizes)).run()
    Scene(groups, 8, 2, 64, 64, seed=sum(sizes)).run()


@pytest.mark.parametrize("sizes", [(1,) * 60 + (150,), (1,) * 30 + (80, 1, 1, 90) + (2,) * 20,
                                   (100, 90) + (1,) * 66])
@pytest.mark.parametrize("hq,hkv,d", [(4, 1, 128), (16, 4, 64)])
def test_large_groups_among_small_ones(sizes, hq, hkv, d):
    """Partial results of a large group lie within the workspace whatever its number, and the
    call writes nothing behind it."""
    s = Scene([(100 + i, [1 + (11 * j) % 40 for j in range(n)]) for i, n in enumerate(sizes)],
              hq, hkv, d, 32, seed=len(sizes))
    q, c, b = s.queries(1), s.cache(), s.batch(1)
    n = s.fpx.decode_workspace_size(c, b)
    ws = torch.full((8 * n,), 0x5A, dtype=torch.uint8, device="cuda")
    s.check(q, s.fpx.decode_attn(_dev(q), c, 0, b, workspace=ws[:n]), 1)
    assert bool((ws[n:] == 0x5A).all())


def test_a_long_prefix_of_many_rows():
    Scene([(40000, [3, 200] * 40)], 4, 1, 128, 128, seed=21).run()


@pytest.mark.parametrize("d", [64, 128])
def test_several_groups(d):
    groups = [(200, [3, 70]), (0, [5, 100, 1]), (77, [30]), (1000, [20, None, 64, 21]),
              (50, [None, None]), (64, [1, None])]
    Scene(groups, 8, 2, d, 16, seed=d).run(2)


@pytest.mark.parametrize("nq", [5, 16])
def test_groups_of_fewer_tokens_than_queries(nq):
    """A sequence with more queries than tokens leaves its group no prefix to share."""
    Scene([(3, [0, 1, 30]), (40, [2, 9]), (0, [1, 2]), (2, [0, None])], 4, 2, 64, 16,
          seed=nq).run(nq)


@pytest.mark.parametrize("seed", range(10))
def test_random_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    hkv = int(rng.integers(1, 4))
    groups = []
    for _ in range(rng.integers(1, 9)):
        own = [None if rng.random() < 0.1 else int(np.exp(rng.uniform(0, 6.2)))
               for _ in range(rng.integers(1, 30))]
        groups.append((0 if rng.random() < 0.3 else int(np.exp(rng.uniform(1, 6.8))), own))
    Scene(groups, hkv * int(rng.integers(1, 9)), hkv, int(rng.choice([64, 128])),
          int(rng.choice([16, 32, 64, 128, 256])), seed=seed).run(int(rng.choice([1, 1, 2, 7])))


def test_a_sequence_shorter_than_the_prefix():
    """The group then shares what all of its queries see."""
    s = Scene([(300, [5, 9, 40])], 4, 1, 64, 32, seed=5)
    n = 130
    s.meta[s.lens_at + s.slots[1]] = n
    s.seqs[1] = (s.seqs[1][0][:n], s.seqs[1][1][:n])
    s.run(4)


def test_shared_and_not_shared_agree():
    s = Scene([(500, [30, 31, 32, 200])], 8, 2, 128, 64, seed=6)
    q = s.queries(1)
    c = s.cache()
    a = s.fpx.decode_attn(_dev(q), c, 0, s.batch(1))
    b = s.fpx.decode_attn(_dev(q), c, 0, s.batch(1, shared=False))
    s.check(q, a, 1)
    s.check(q, b, 1)


def test_repeatable():
    s = Scene([(3000, [100, 1, 64, 900]), (0, [5000, 40])], 8, 2, 128, 64, seed=7)
    q, c, b = _dev(s.queries(2)), s.cache(), s.batch(2)
    first = s.fpx.decode_attn(q, c, 0, b)
    for _ in range(5):
        assert torch.equal(first, s.fpx.decode_attn(q, c, 0, b))


@pytest.mark.parametrize("scale", [1e-4, 0.02, 1.0, 8.0])
def test_softmax_scale(scale):
    Scene([(90, [7, 40])], 4, 1, 64, 16, seed=8).run(1, True, scale)


@pytest.mark.parametrize("spread", [0.0, 30.0])
def test_flat_and_peaked_scores(spread):
    """All scores equal, and one key with all the weight."""
    Scene([(257, [1, 300])], 4, 1, 128, 64, seed=9, spread=spread).run()


@pytest.mark.parametrize("gain", [1e-30, 1e30])
def test_size_of_values(gain):
    Scene([(64, [1, 300])], 4, 1, 64, 64, seed=10, gain=gain).run()


INF, NINF, NAN, LOWEST = 0x7F80, 0xFF80, 0x7FC0, 0xFF7F


@pytest.mark.parametrize("pattern", [INF, NINF, NAN])
@pytest.mark.parametrize("d", [64, 128])
def test_odd_values_of_later_tokens(pattern, d):
    """Drafts whose values are infinite or NaN: the queries before them do not see them, the
    ones at and after them do, as the formula has it."""
    nq = 5
    for n in (5, 64, 66, 130, 4):
        s = Scene([(0, [n, n + 7]), (100, [n, n + 30])], 4, 1, d, 16, seed=n)
        for b in (0, 3):
            m = len(s.seqs[b][0])
            v = bits(s.rng.standard_normal((1, d)))
            v[:, 1::3] = pattern
            s.put(b, m - 2, v=v)
        s.run(nq)


@pytest.mark.parametrize("pattern", [INF, NAN])
def test_odd_keys_of_later_tokens(pattern):
    s = Scene([(64, [70, 10])], 2, 1, 64, 32, seed=12)
    for b in (0, 1):
        k = bits(s.rng.standard_normal((1, 64)))
        k[:, 5] = pattern
        s.put(b, len(s.seqs[b][0]) - 1, k=k)
    q = s.queries(4)
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(4))
    got = floats(o.view(torch.int16).cpu().numpy().view(np.uint16)).reshape(2, 4, 2, 64)
    for b, (k, v) in enumerate(s.seqs):
        want, mass = attend(floats(q[b * 4:b * 4 + 3]), floats(k[:-1]), floats(v[:-1]), 0.125)
        assert np.all(np.abs(got[b, :3] - want) <= tolerance(want, mass))


@pytest.mark.parametrize("pattern", [INF, NAN])
@pytest.mark.parametrize("n", [1, 3, 200])
def test_odd_keys_come_through(pattern, n):
    """A visible key that is NaN, or whose score is +inf, makes its queries NaN, whether it is
    the only one of its range of keys or not; other sequences and KV heads stay as they are."""
    s = Scene([(48, [n, 20]), (0, [n])], 4, 2, 64, 16, seed=n)
    q = bits(np.abs(floats(s.queries(1))) + 0.1)
    for b in (0, 2):
        k = np.array(s.seqs[b][0][-1])
        k[0, 3] = pattern
        s.put(b, len(s.seqs[b][0]) - 1, k=k)
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(1))
    assert bool(torch.isnan(o[[0, 2]][:, :2].float()).all())
    s.check(q, o, 1)


def test_scores_of_minus_infinity():
    """Keys whose scores are -inf have no weight; a query with no other key gets 0."""
    s = Scene([(0, [40, 3])], 2, 1, 64, 16, seed=13)
    q = np.abs(floats(s.queries(1)))
    k = np.zeros((1, 64), np.uint16)
    k[:, 0] = NINF
    for t in (0, 7, 39):
        s.put(0, t, k=k)
    for t in range(3):
        s.put(1, t, k=k)
    q = bits(q + 0.1)
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(1))
    s.check(q, o, 1)
    assert not o[1].any()


def test_largest_finite_scores():
    s = Scene([(0, [40])], 2, 1, 64, 16, seed=14)
    k = np.full((1, 64), LOWEST, np.uint16)
    s.put(0, 3, k=k)
    q = bits(np.full((1, 2, 64), 1.0))
    o = s.fpx.decode_attn(_dev(q), s.cache(), 0, s.batch(1))
    s.check(q, o, 1)


def test_strided_queries_and_buffers():
    s = Scene([(128, [9, 77, 31])], 6, 2, 128, 64, seed=15)
    q = s.queries(2)
    wide = torch.full((6, 10, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :6] = _dev(q)
    c, b = s.cache(), s.batch(2)
    out = torch.full((6, 6, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    n = s.fpx.decode_workspace_size(c, b)
    ws = torch.full((n + 256,), 255, dtype=torch.uint8, device="cuda")
    got = s.fpx.decode_attn(wide[:, :6], c, 0, b, out=out, workspace=ws[:n])
    assert got is out
    s.check(q, out, 2)
    assert bool((ws[n:] == 255).all())


def test_layers_and_offsets_past_32_bits():
    """The second layer of a pool of over 2^31 elements, pages at its far end."""
    import paper_2502_20766_amd as fpx
    pages, hkv, d, page, n = 9000, 8, 128, 128, 500
    c = fpx.Cache(2, pages, hkv, d, 2, pages, page)
    fpx.cache_reserve(c, [0], [(pages - 5) * page])
    fpx.cache_reserve(c, [1], [n])
    g = torch.Generator("cuda").manual_seed(3)
    k = torch.randn(n, hkv, d, generator=g, device="cuda").bfloat16()
    v = torch.randn(n, hkv, d, generator=g, device="cuda").bfloat16()
    q = torch.randn(1, 16, d, generator=g, device="cuda").bfloat16()
    fpx.cache_write(c, 1, k, v, [1], [0, n])
    c.check()
    o = fpx.decode_attn(q, c, 1, fpx.DecodeBatch([1], 16))
    host = lambda x: floats(x.view(torch.int16).cpu().numpy().view(np.uint16))  # noqa: E731
    want, mass = attend(host(q), host(k), host(v), 1 / math.sqrt(d))
    assert np.all(np.abs(host(o) - want) <= tolerance(want, mass))


def test_a_long_sequence():
    """300k tokens, all of them the work of one KV head: hundreds of pieces to join."""
    Scene([(0, [300001])], 2, 1, 64, 256, seed=16).run()


def test_on_another_stream():
    s = Scene([(128, [9, 77])], 4, 1, 64, 64, seed=17)
    q = s.queries(1)
    dq, c, b = _dev(q), s.cache(), s.batch(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o = s.fpx.decode_attn(dq, c, 0, b, stream=side)
    side.synchronize()
    s.check(q, o, 1)


def test_decoding_loop_in_a_graph():
    """Steps captured once and replayed: lengths, new pages and copies of shared pages follow the
    device's state, each replay like the eager call from the same state."""
    import paper_2502_20766_amd as fpx
    hq, hkv, d, page, layers, B = 8, 2, 64, 16, 2, 3
    g = torch.Generator("cuda").manual_seed(11)
    prompt = 45

    def fresh():
        c = fpx.Cache(layers, 60, hkv, d, 4, 12, page)
        gg = torch.Generator("cuda").manual_seed(12)
        c.k.zero_(), c.v.zero_()
        fpx.cache_reserve(c, [0], [prompt])
        for layer in range(layers):
            k = torch.randn(prompt, hkv, d, generator=gg, device="cuda").bfloat16()
            v = torch.randn(prompt, hkv, d, generator=gg, device="cuda").bfloat16()
            fpx.cache_write(c, layer, k, v, [0], [0, prompt])
        fpx.cache_fork(c, [0, 0], [1, 2])
        return c

    slots, cu = np.arange(B, dtype=np.int32), np.arange(B + 1, dtype=np.int32)
    batch = fpx.DecodeBatch(slots, hq, 1, [0, B], [prompt])
    eager, live = fresh(), fresh()
    ws = torch.empty(fpx.cache_workspace_size(live), dtype=torch.uint8, device="cuda")
    dws = torch.empty(fpx.decode_workspace_size(live, batch), dtype=torch.uint8, device="cuda")
    x = torch.randn(B, hq + 2 * hkv, d, generator=g, device="cuda").bfloat16()
    outs = [torch.empty(B, hq, d, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]

    def step(c, o):
        fpx.cache_reserve(c, slots, 1, workspace=ws)
        for layer in range(layers):
            fpx.cache_write(c, layer, x[:, hq:hq + hkv], x[:, hq + hkv:], slots, cu)
            fpx.decode_attn(x[:, :hq], c, layer, batch, out=o[layer], workspace=dws)

    torch.cuda.synchronize()
    before = live.meta.clone(), live.k.clone(), live.v.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(live, outs)
    live.meta.copy_(before[0]), live.k.copy_(before[1]), live.v.copy_(before[2])
    for i in range(25):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        graph.replay()
        want = [torch.empty_like(o) for o in outs]
        step(eager, want)
        torch.cuda.synchronize()
        assert torch.equal(live.meta, eager.meta), i
        assert torch.equal(live.k, eager.k) and torch.equal(live.v, eager.v), i
        for a, b in zip(outs, want):
            assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all()), i
    live.check()


@pytest.mark.parametrize("make", [lambda n: torch.empty(n, dtype=torch.uint8),
                                  lambda n: torch.empty(n, dtype=torch.int32, device="cuda"),
                                  lambda n: torch.empty(2 * n, dtype=torch.uint8,
                                                        device="cuda")[::2]])
def test_refuses_workspaces_that_are_not_bytes_on_the_gpu(make):
    s = Scene([(0, [5])], 4, 1, 64, 16, seed=18)
    c, b = s.cache(), s.batch(1)
    with pytest.raises(ValueError):
        s.fpx.decode_attn(_dev(s.queries(1)), c, 0, b,
                          workspace=make(s.fpx.decode_workspace_size(c, b)))
    n = s.fpx.cache_workspace_size(c)
    with pytest.raises(ValueError):
        s.fpx.cache_reserve(c, [0], 1, workspace=make(n))
    with pytest.raises(ValueError):
        s.fpx.cache_compact(c, workspace=make(n))


@pytest.mark.parametrize("bad", ["dtype", "rows", "heads", "out", "workspace", "layer"])
def test_refusals(bad):
    s = Scene([(0, [5])], 4, 1, 64, 16, seed=18)
    c, b = s.cache(), s.batch(1)
    q = _dev(s.queries(1))
    kw, layer = {}, 0
    if bad == "dtype":
        q = q.float()
    elif bad == "rows":
        q = torch.cat([q, q])
    elif bad == "heads":
        q = q[:, :2].contiguous()
    elif bad == "out":
        kw["out"] = torch.empty(1, 4, 128, dtype=torch.bfloat16, device="cuda")
    elif bad == "workspace":
        kw["workspace"] = torch.empty(16, dtype=torch.uint8, device="cuda")
    else:
        layer = 1
    with pytest.raises((ValueError, s.fpx.FlexPrefillError)):
        s.fpx.decode_attn(q, c, layer, b, **kw)
