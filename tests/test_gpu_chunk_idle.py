"""chunk_attn beside sequences without tokens that have many rows: zeros for those, the others as they are
alone, whatever records an earlier batch has left in the workspace."""
import numpy as np
import pytest

from test_gpu_chunk import Chunks, _dev
from test_gpu_decode import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# (query heads, KV heads, head dim, tokens, queries, the first record that no part of the call has,
# and records): more segments than records, few parts, and workgroups of every XCD left over
FEW_PARTS = [(32, 2, 128, [None, None, 1207], [995, 995, 1], 80, 85),
             (32, 2, 64, [1479, None], [39, 3037], 152, 153),
             (32, 2, 64, [1241, 0], [41, 3078], 80, 85),
             (8, 2, 128, [1151, None, 0], [1, 5538, 2462], 80, 85)]


@pytest.mark.parametrize("hq,hkv,d,lens,news,first,records", FEW_PARTS)
def test_a_workspace_of_an_earlier_batch(hq, hkv, d, lens, news, first, records):
    s = Chunks(lens, news, hq, hkv, d, 64, seed=first)
    q, c, b = s.q_bits(), s.cache(), s.of()
    ws = torch.zeros(s.fpx.chunk_workspace_size(c, b), dtype=torch.uint8, device="cuda")
    # records as another batch leaves them: a segment of two pieces, whose rows the call has too
    at = ws[:16 * records].view(torch.int32).view(records, 4)
    busy = int(np.argmax([n or 0 for n in lens]))
    at[:] = torch.tensor([2 | 3 << 16, busy, 0, 0], dtype=torch.int32)
    o = s.fpx.chunk_attn(_dev(q), c, 0, b, workspace=ws)
    s.verify(q, o)
    assert not bool(at[first:].any())


def test_a_workspace_of_another_call():
    """The same after a call that cuts long sequences, and that call again after it."""
    few = Chunks([None, None, 1207], [995, 995, 1], 32, 2, 128, 64, seed=3)
    long = Chunks([9000, 3000, 6001], [700, 1, 600], 32, 2, 128, 64, seed=4)
    calls = [(s, s.q_bits(), s.cache(), s.of()) for s in (few, long)]
    size = max(s.fpx.chunk_workspace_size(c, b) for s, _, c, b in calls)
    ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
    for i in (1, 0, 1, 0):
        s, q, c, b = calls[i]
        s.verify(q, s.fpx.chunk_attn(_dev(q), c, 0, b, workspace=ws))


def test_a_graph_whose_sequences_are_emptied(gpu):  # noqa: F811
    """Captured while all sequences have tokens; replayed, and in between two of them freed."""
    g = torch.Generator("cuda").manual_seed(1)
    hq, hkv, d, cu = 32, 2, 128, [0, 995, 1990, 1991]
    c = gpu.Cache(1, 60, hkv, d, 3, 20, 64)
    kv = torch.randn(2, 3207, hkv, d, generator=g, device="cuda").bfloat16()

    def fill(slots):
        at = [[0, 1000, 2000, 3207][s:s + 2] for s in slots]
        gpu.cache_reserve(c, slots, [b - a for a, b in at])
        rows = torch.cat([torch.arange(a, b) for a, b in at]).cuda()
        gpu.cache_write(c, 0, kv[0, rows], kv[1, rows], slots, np.cumsum([0] + [b - a for a, b in at]))

    fill([0, 1, 2])
    q = torch.randn(1991, hq, d, generator=g, device="cuda").bfloat16()
    b, out = gpu.ChunkBatch([0, 1, 2], cu, hq), torch.empty_like(q)
    ws = torch.empty(gpu.chunk_workspace_size(c, b), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gpu.chunk_attn(q, c, 0, b, out=out, workspace=ws)
    for full in (True, False, False, True, False):
        if not full:
            gpu.cache_free(c, [0, 1])
        out.fill_(5.0)
        graph.replay()
        want = gpu.chunk_attn(q, c, 0, b)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert bool(out[:1990].any()) == full and bool(out[1990:].any())
        if not full:
            fill([0, 1])
    c.check()


@pytest.mark.parametrize("seed", range(12))
def test_drawn_batches_with_idle_sequences(seed):
    """Sequences without a slot or without tokens, some of thousands of rows, beside others of drawn
    lengths."""
    rng = np.random.default_rng(200 + seed)
    hkv = int(rng.choice([1, 2, 2, 4]))
    hq, d = hkv * int(rng.choice([1, 4, 7, 16])), int(rng.choice([64, 128]))
    n = int(rng.integers(2, 8))
    lens = [[None, 0, int(2 ** rng.uniform(0, 12.5))][int(rng.integers(0, 3))] for _ in range(n)]
    lens[int(rng.integers(0, n))] = 1200 + int(rng.integers(0, 6000))
    news = [int(2 ** rng.uniform(0, 12)) if not x else min(x, int(2 ** rng.uniform(0, 8))) for x in lens]
    s = Chunks(lens, news, hq, hkv, d, int(rng.choice([16, 64, 256])), seed=seed)
    q, c, b = s.q_bits(), s.cache(), s.of()
    ws = torch.zeros(s.fpx.chunk_workspace_size(c, b), dtype=torch.uint8, device="cuda")
    for _ in range(2):
        s.verify(q, s.fpx.chunk_attn(_dev(q), c, 0, b, workspace=ws))
