"""The paged cache's operators together, as a serving loop calls them: prompts appended chunk by chunk
and attended to, decoding after them, the sparse prefill of rotated heads; captured into graphs, on
other streams, and where offsets pass 32 bits."""
import numpy as np
import pytest

from chunk_model import chunk_attend, chunk_tolerance
from test_gpu_decode import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()


def host(x):
    return x.double().cpu().numpy()


def close(o, q, k, v):
    """o of the last queries q over k and v (what the cache holds), all bf16 on the GPU."""
    want, mass = chunk_attend(host(q), host(k), host(v), q.shape[2] ** -0.5)
    assert np.all(np.abs(host(o) - want) <= chunk_tolerance(want, mass))


def model_of(fpx, d, norm, layout="half"):
    g = torch.Generator("cuda").manual_seed(d)
    w = (1 + 0.2 * torch.randn(2, d, generator=g, device="cuda")).bfloat16()
    return (fpx.Rope(d, base=1e5, layout=layout, scaling="parts", factor=4.0, original_len=256),
            fpx.HeadNorm(w[0], w[1]) if norm else None)


@pytest.mark.parametrize("hq,hkv,d,page,layout,norm", [
    (8, 2, 128, 64, "half", True), (4, 4, 64, 16, "interleaved", False), (7, 1, 64, 128, "half", True),
    (16, 1, 128, 32, "interleaved", True)])
def test_prompts_in_chunks_then_decoding(gpu, hq, hkv, d, page, layout, norm):     # noqa: F811
    fpx, layers = gpu, 2
    g = torch.Generator("cuda").manual_seed(1)
    rope, weights = model_of(fpx, d, norm, layout)
    c = fpx.Cache(layers, 3 * (1024 // page) + 8, hkv, d, 5, 1024 // page, page)
    slots = [3, 0, 4]
    kept = {(s, layer): [] for s in slots for layer in range(layers)}
    done = dict.fromkeys(slots, 0)
    for counts in ([300, 1, 64], [1, 77, 0], [129, 1, 1], [1, 1, 1], [200, 200, 200]):
        cu = np.cumsum([0] + counts)
        fpx.cache_reserve(c, slots, counts)
        batch = fpx.ChunkBatch(slots, cu, hq)
        at = np.concatenate([done[s] + np.arange(n) for s, n in zip(slots, counts)])
        at = torch.from_numpy(at.astype(np.int32)).cuda()
        for layer in range(layers):
            x = randn(g, int(cu[-1]), hq + 2 * hkv, d)
            q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
            qr, kr = fpx.rotate(q, k, at, rope, weights)
            qa = fpx.cache_append(c, layer, q, k, v, slots, cu, rope, weights)
            assert torch.equal(qa, qr)           # positions from the cache are those of the caller
            o = fpx.chunk_attn(qa, c, layer, batch)
            for i, s in enumerate(slots):
                kept[s, layer].append((kr[cu[i]:cu[i + 1]], v[cu[i]:cu[i + 1]]))
                k1, v1 = (torch.cat(y) for y in zip(*kept[s, layer]))
                close(o[cu[i]:cu[i + 1]], qr[cu[i]:cu[i + 1]], k1, v1)
        for s, n in zip(slots, counts):
            done[s] += n
    # a fork, then a step in which the copies go on apart, by decode_attn and chunk_attn alike
    fpx.cache_fork(c, [3], [1])
    slots = [3, 1]
    fpx.cache_reserve(c, slots, 1)
    x = randn(g, 2, hq + 2 * hkv, d)
    at = torch.full((2,), done[3], dtype=torch.int32, device="cuda")
    for layer in range(layers):
        q, kr = fpx.rotate(x[:, :hq], x[:, hq:hq + hkv], at, rope, weights)
        qa = fpx.cache_append(c, layer, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], slots, [0, 1, 2],
                              rope, weights)
        assert torch.equal(q, qa)
        a = fpx.chunk_attn(qa, c, layer, fpx.ChunkBatch(slots, [0, 1, 2], hq))
        b = fpx.decode_attn(qa, c, layer, fpx.DecodeBatch(slots, hq, 1, [0, 2], [done[3]]))
        k1, v1 = (torch.cat(y) for y in zip(*kept[3, layer]))
        for i in range(2):
            for o in (a, b):
                close(o[i:i + 1], q[i:i + 1], torch.cat([k1, kr[i:i + 1]]),
                      torch.cat([v1, x[i:i + 1, hq + hkv:]]))
    c.check()


def test_sparse_prefill_of_rotated_heads(gpu):     # noqa: F811
    """rotate before select and sparse_attn; with the whole weight kept they are chunk_attn of the
    same prompt from the cache."""
    fpx, hq, hkv, d = gpu, 8, 2, 128
    g = torch.Generator("cuda").manual_seed(2)
    rope, weights = model_of(fpx, d, True)
    cu = [0, 700, 1000]
    x = randn(g, 1000, hq + 2 * hkv, d)
    q, k, v = x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]
    at = torch.cat([torch.arange(700), torch.arange(300)]).to(torch.int32).cuda()
    qr, kr = fpx.rotate(q, k, at, rope, weights)
    idx = fpx.select(qr, kr, cu, gamma=1.0, tau=0.1)
    sparse = fpx.sparse_attn(qr, kr, v.contiguous(), idx)
    c = fpx.Cache(1, 40, hkv, d, 2, 20, 64)
    fpx.cache_reserve(c, [1, 0], [700, 300])
    qa = fpx.cache_append(c, 0, q, k, v, [1, 0], cu, rope, weights)
    assert torch.equal(qa, qr)
    o = fpx.chunk_attn(qa, c, 0, fpx.ChunkBatch([1, 0], cu, hq))
    for a, b in ((0, 700), (700, 1000)):
        close(sparse[a:b], qr[a:b], kr[a:b], v[a:b])
        close(o[a:b], qr[a:b], kr[a:b], v[a:b])


class Loop:
    """Steps of a loop over its own cache, alike for the same seed."""

    def __init__(self, fpx, counts, hq, hkv, d, first=None, max_pages=40):
        self.fpx, self.hq, self.hkv, self.d, self.layers = fpx, hq, hkv, d, 2
        g = torch.Generator("cuda").manual_seed(3)
        n = len(counts)
        self.c = fpx.Cache(self.layers, max_pages * n, hkv, d, n, max_pages, 16)
        self.c.k.zero_(), self.c.v.zero_()
        self.rope, self.norm = model_of(fpx, d, True)
        self.slots, self.counts = np.arange(n, dtype=np.int32), np.array(counts, np.int32)
        self.cu = np.cumsum([0] + list(counts)).astype(np.int32)
        self.batch = fpx.ChunkBatch(self.slots, self.cu, hq)
        first = first or [45 + 30 * i for i in range(n)]
        cu = np.cumsum([0] + first)
        fpx.cache_reserve(self.c, self.slots, first)
        for layer in range(self.layers):
            x = randn(g, int(cu[-1]), 2 * hkv, d)
            fpx.cache_append(self.c, layer, None, x[:, :hkv], x[:, hkv:], self.slots, cu, self.rope,
                             self.norm)
        T = int(self.cu[-1])
        self.x = torch.zeros(T, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
        self.q = torch.zeros(T, hq, d, dtype=torch.bfloat16, device="cuda")
        self.o = [torch.zeros_like(self.q) for _ in range(self.layers)]
        sizes = fpx.cache_workspace_size(self.c), fpx.chunk_workspace_size(self.c, self.batch)
        self.ws = [torch.empty(s, dtype=torch.uint8, device="cuda") for s in sizes]

    def step(self):
        hq, hkv, x = self.hq, self.hkv, self.x
        self.fpx.cache_reserve(self.c, self.slots, self.counts, workspace=self.ws[0])
        for layer in range(self.layers):
            self.fpx.cache_append(self.c, layer, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:],
                                  self.slots, self.cu, self.rope, self.norm, q_out=self.q)
            self.fpx.chunk_attn(self.q, self.c, layer, self.batch, out=self.o[layer],
                                workspace=self.ws[1])

    def capture(self):
        before = self.c.meta.clone(), self.c.k.clone(), self.c.v.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step()
        torch.cuda.synchronize()
        self.c.meta.copy_(before[0]), self.c.k.copy_(before[1]), self.c.v.copy_(before[2])
        return graph

    def same(self, other):
        assert torch.equal(self.c.meta, other.c.meta)
        assert torch.equal(self.c.k, other.c.k) and torch.equal(self.c.v, other.c.v)
        assert torch.equal(self.q, other.q)
        for a, b in zip(self.o, other.o):
            assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("d", [64, 128])
def test_two_graphs_of_steps_that_share_their_workspaces(gpu, d):     # noqa: F811
    """Lengths and pages follow the device's state from replay to replay; each replay is, to the bit,
    the eager step from the same state, though another graph used the workspaces in between."""
    live = [Loop(gpu, [5, 1, 0, 9], 8, 2, d), Loop(gpu, [17, 1], 8, 2, d)]
    both = [max((a, b), key=lambda t: t.numel()) for a, b in zip(live[0].ws, live[1].ws)]
    live[0].ws = live[1].ws = both
    eager = [Loop(gpu, [5, 1, 0, 9], 8, 2, d), Loop(gpu, [17, 1], 8, 2, d)]
    graphs = [a.capture() for a in live]
    g = torch.Generator("cuda").manual_seed(4)
    for i in range(14):
        for a, b, graph in zip(live, eager, graphs):
            x = randn(g, *a.x.shape)
            a.x.copy_(x), b.x.copy_(x)
            graph.replay()
        for a, b in zip(live, eager):
            b.step()
            torch.cuda.synchronize()
            a.same(b)
    for a in live:
        a.c.check()


@pytest.mark.parametrize("d", [64, 128])
def test_a_graph_whose_sequences_become_long(gpu, d):     # noqa: F811
    """Captured while row tiles stay whole, replayed beyond the lengths at which they are cut."""
    make = lambda: Loop(gpu, [30, 1, 0], 4, 2, d, [800, 880, 5], 90)     # noqa: E731
    live, eager = make(), make()
    graph = live.capture()
    g = torch.Generator("cuda").manual_seed(8)
    for i in range(20):
        x = randn(g, *live.x.shape)
        live.x.copy_(x), eager.x.copy_(x)
        graph.replay()
        eager.step()
        torch.cuda.synchronize()
        live.same(eager)
    live.c.check()


def test_rotate_in_a_graph(gpu):     # noqa: F811
    g = torch.Generator("cuda").manual_seed(5)
    rope, norm = model_of(gpu, 128, True, "interleaved")
    x, at = randn(g, 300, 6, 128), torch.arange(300, dtype=torch.int32, device="cuda")
    q, k = torch.empty_like(x[:, :4]).contiguous(), torch.empty_like(x[:, 4:]).contiguous()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gpu.rotate(x[:, :4], x[:, 4:], at, rope, norm, q, k)
        q2, k2 = gpu.rotate(x[:, :4], x[:, 4:], at, rope, norm)
    for i in range(4):
        x.copy_(randn(g, *x.shape)), at.add_(1000 * i)
        graph.replay()
        want = gpu.rotate(x[:, :4], x[:, 4:], at, rope, norm)
        torch.cuda.synchronize()
        for a, b in zip((q, k, q2, k2), want * 2):
            assert torch.equal(a, b)


def test_a_step_on_another_stream(gpu):     # noqa: F811
    """Calls that name a stream run there, outputs and workspaces that they allocate belong to it."""
    g = torch.Generator("cuda").manual_seed(6)
    rope, norm = model_of(gpu, 128, True)
    c = gpu.Cache(1, 60, 2, 128, 2, 30, 32)
    side = torch.cuda.Stream()
    kept = []
    for n in (90, 1, 40):
        x = randn(g, n, 8, 128)
        at = torch.arange(n, dtype=torch.int32, device="cuda") + sum(len(k) for k, _ in kept)
        side.wait_stream(torch.cuda.current_stream())
        gpu.cache_reserve(c, [1], n, stream=side)
        q, k = gpu.rotate(x[:, :4], x[:, 4:6], at, rope, norm, stream=side)
        qa = gpu.cache_append(c, 0, x[:, :4], x[:, 4:6], x[:, 6:], [1], [0, n], rope, norm, stream=side)
        o = gpu.chunk_attn(qa, c, 0, gpu.ChunkBatch([1], [0, n], 4), stream=side)
        side.synchronize()
        kept.append((k, x[:, 6:]))
        assert torch.equal(q, qa)
        close(o, q, *(torch.cat(y) for y in zip(*kept)))


def test_offsets_past_32_bits(gpu):     # noqa: F811
    """A layer whose pages lie more than 2^31 elements into the pool; rows of a projection too."""
    hq, hkv, d, layers = 8, 4, 128, 40
    g = torch.Generator("cuda").manual_seed(7)
    c = gpu.Cache(layers, 2000, hkv, d, 2, 20, 64)
    assert c.k.numel() > 2 ** 31
    rope, norm = model_of(gpu, d, True)
    x = randn(g, 700, hq + 2 * hkv, d)
    at = torch.arange(700, dtype=torch.int32, device="cuda")
    q, k = gpu.rotate(x[:, :hq], x[:, hq:hq + hkv], at, rope, norm)
    gpu.cache_reserve(c, [1], 700)
    qa = gpu.cache_append(c, layers - 1, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], [1], [0, 700],
                          rope, norm)
    assert torch.equal(q, qa)
    close(gpu.chunk_attn(qa, c, layers - 1, gpu.ChunkBatch([1], [0, 700], hq)), q, k, x[:, hq + hkv:])
    # (the same from queries of which the last lie past 2^31 elements)
    del c
    T, wide = 110000, 20480
    big = torch.empty(T, wide, dtype=torch.bfloat16, device="cuda")
    assert (T - 300) * wide > 2 ** 31
    rows = big[:, :hq * d].view(T, hq, d)
    rows.zero_()
    rows[-300:].copy_(x[:300, :hq])
    at = torch.zeros(T, dtype=torch.int32, device="cuda")
    at[-300:] = torch.arange(300, dtype=torch.int32, device="cuda")
    out, _ = gpu.rotate(rows, None, at, rope, norm)
    assert torch.equal(out[-300:], q[:300]) and not bool(out[:-300].any())
    same, _ = gpu.rotate(rows, None, at, rope, norm, q_out=rows)
    assert torch.equal(same[-300:], q[:300])
    c = gpu.Cache(1, 16, hkv, d, 256, 16, 64)
    gpu.cache_reserve(c, [1], 300)
    gpu.cache_append(c, 0, None, x[:300, hq:hq + hkv], x[:300, hq + hkv:], [1], [0, 300], rope, norm)
    o = gpu.chunk_attn(rows, c, 0, gpu.ChunkBatch([-1, 1], [0, T - 300, T], hq))
    close(o[-300:], q[:300], k[:300], x[:300, hq + hkv:])
    assert not bool(o[:-300].any())


@pytest.mark.parametrize("seed", range(10))
def test_drawn_batches(gpu, seed):     # noqa: F811
    """Batches of drawn lengths, heads and pages, among them several long chunks at once, for which the
    kernel pairs row tiles in more than one way."""
    from test_gpu_chunk import Chunks
    rng = np.random.default_rng(100 + seed)
    hkv = int(rng.integers(1, 4))
    hq, d = hkv * int(rng.integers(1, 9)), int(rng.choice([64, 128, 128]))
    n = int(rng.integers(2, 14))
    lens = [int(2 ** rng.uniform(0, 11.5)) for _ in range(n)]
    news = [int(min(x + 1, 2 ** rng.uniform(0, 10.5))) if rng.random() < 0.8 else 0 for x in lens]
    if seed % 2:
        news = [x if rng.random() < 0.6 else 1 for x in lens]       # whole prompts and single tokens
    Chunks(lens, news, hq, hkv, d, int(rng.choice([16, 32, 64, 128, 256])), seed=seed).go()
