"""The cache's bookkeeping and copies against the host model, call by call and bit for bit."""
import numpy as np
import pytest

from cache_model import FULL, SHARED, TOO_LONG, Model

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_20766_amd as fpx
    fpx.lib()
    return fpx


class Pair:
    """A cache on the GPU and the model of it; every call goes to both."""

    def __init__(self, layers=2, pages=40, hkv=2, d=64, slots=6, max_pages=12, page=16, seed=0):
        import paper_2502_20766_amd as fpx
        self.fpx, self.rng = fpx, np.random.default_rng(seed)
        self.dims = (layers, hkv, d)
        self.m = Model(layers, pages, hkv, d, slots, max_pages, page)
        self.c = fpx.Cache(layers, pages, hkv, d, slots, max_pages, page)
        # what the pools held before must not matter, and must stay where nothing is written
        self.m.k[:] = self.rng.integers(0, 65536, self.m.k.shape, dtype=np.uint16)
        self.m.v[:] = self.rng.integers(0, 65536, self.m.v.shape, dtype=np.uint16)
        self.c.k.copy_(self._dev(self.m.k))
        self.c.v.copy_(self._dev(self.m.v))

    @staticmethod
    def _dev(x):
        return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)

    def reserve(self, slots, counts):
        self.fpx.cache_reserve(self.c, slots, counts)
        self.m.reserve(slots, counts)

    def write(self, slots, counts, stride=None):
        layers, hkv, d = self.dims
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        for layer in range(layers):
            k = self.rng.integers(0, 65536, (cu[-1], hkv, d), dtype=np.uint16)
            v = self.rng.integers(0, 65536, (cu[-1], hkv, d), dtype=np.uint16)
            self.m.write(layer, k, v, slots, cu)
            both = np.zeros((cu[-1], 2 * hkv + 1, d), np.uint16)   # rows with a stride
            both[:, :hkv], both[:, hkv + 1:] = k, v
            x = self._dev(both)
            self.fpx.cache_write(self.c, layer, x[:, :hkv], x[:, hkv + 1:], slots, cu)

    def append(self, slots, counts):
        self.reserve(slots, counts)
        self.write(slots, counts)

    def fork(self, src, dst):
        self.fpx.cache_fork(self.c, src, dst)
        self.m.fork(src, dst)

    def truncate(self, slots, lens):
        self.fpx.cache_truncate(self.c, slots, lens)
        self.m.truncate(slots, lens)

    def free(self, slots):
        self.fpx.cache_free(self.c, slots)
        self.m.truncate(slots, [0] * len(slots))

    def compact(self):
        self.fpx.cache_compact(self.c)
        self.m.compact()

    def same(self, what=""):
        assert np.array_equal(self.c.meta.cpu().numpy(), self.m.meta()), what
        for a, b in ((self.c.k, self.m.k), (self.c.v, self.m.v)):
            assert np.array_equal(a.view(torch.int16).cpu().numpy().view(np.uint16), b), what


@pytest.mark.parametrize("d,hkv,page", [(64, 2, 16), (128, 1, 64), (128, 8, 128), (64, 3, 256)])
@pytest.mark.parametrize("counts", [[1, 1, 1], [0, 5, 0], [16, 17, 15], [63, 64, 65],
                                    [200, 1, 33]])
def test_append_twice(d, hkv, page, counts):
    p = Pair(pages=80, hkv=hkv, d=d, page=page, max_pages=40, seed=page + counts[0])
    p.append([4, 0, 2], counts)
    p.same("first")
    p.append([2, 4, 0], counts)          # starts inside steps, units and pages
    p.same("second")
    p.append([0, 5], [1, 7])
    p.same("third")


def test_a_step_of_every_slot():
    p = Pair(layers=1, pages=600, slots=256, max_pages=4, seed=3)
    lens = np.arange(256) % 33
    p.append(list(range(256)), lens)
    p.append(list(range(255, -1, -1)), [1] * 256)
    p.same()


def test_fork_shares_and_the_last_holder_keeps():
    p = Pair(seed=4)
    p.append([0], [37])                  # three pages, the last not full
    p.fork([0, 0, 0], [1, 2, 3])
    p.same("fork")
    p.append([2, 0, 3, 1], [1, 1, 1, 1])  # slots 2, 0 and 3 copy, slot 1 keeps
    p.same("each its own last page")
    p.fork([2, 2, 0], [4, 1, 5])         # slot 1's pages go back
    p.same("fork over a slot in use")
    p.append([4, 0], [30, 0])            # a count of 0 copies nothing
    p.same("one grows")
    p.free([0, 2])
    p.same("the others still hold the prompt")
    p.free([1, 3, 4, 5])
    p.same("all free")


def test_fork_of_a_full_last_page_copies_nothing():
    p = Pair(seed=5)
    p.append([0], [32])
    p.fork([0], [1])
    p.append([0, 1], [1, 17])
    p.same()


def test_fork_of_an_empty_slot_empties():
    p = Pair(seed=6)
    p.append([1], [20])
    p.fork([0], [1])
    p.same()


def test_truncate_into_a_shared_page():
    p = Pair(seed=7)
    p.append([0], [45])
    p.fork([0], [1])
    p.truncate([1], [19])                # inside a page that slot 0 holds full
    p.same("short")
    p.append([1], [1])                   # so it takes a copy
    p.same("grown again")
    p.truncate([0, 1], [60, 20])         # longer than they are: nothing changes
    p.same("nothing")
    p.truncate([0, 1], [16, 0])
    p.same("whole pages")


def test_many_children_of_one():
    p = Pair(layers=1, pages=700, slots=140, max_pages=6, seed=8)
    p.append([7], [70])
    others = [s for s in range(140) if s != 7]
    p.fork([7] * 139, others)
    p.same("fork")
    p.append(others[:100], [1] * 100)
    p.same("append")
    p.fork([others[i % 3] for i in range(100)], others[30:130])
    p.same("fork again")
    p.free(others)
    p.same("free")


@pytest.mark.parametrize("max_pages", [20, 300, 6000])
@pytest.mark.parametrize("n", [40, 101])
def test_long_lists_and_long_tables(max_pages, n):
    """Forks of several sequences over old ones that share their pages, and lists cut in the
    middle of shared pages, for every length of tables; the last thread's rows not full."""
    p = Pair(1, 2 * max_pages + 3 * n, 1, 64, n + 3, max_pages, 16)
    tokens = 16 * max_pages - 40
    for i in range(3):                   # three sequences, the second one a fork of the first
        if i == 1:
            p.fork([0], [1])
            p.append([1], [20])
        else:
            p.reserve([i], [tokens - 16 * i])
    src = [int(x) for x in p.rng.integers(0, 3, n)]
    dst = [int(x) for x in 3 + p.rng.permutation(n)]
    p.fork(src, dst)
    p.same("fork")
    again = [int(x) for x in p.rng.integers(0, 3, n)]
    p.fork(again, dst)                   # over copies of other sequences
    p.same("fork over forks")
    p.truncate(dst, [int(x) for x in p.rng.integers(0, tokens, n)])
    p.same("truncate")
    p.free([0] + dst[:n // 2])
    p.same("free")


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("pages", [63, 64, 65, 300])
def test_compact(page, pages):
    p = Pair(pages=pages, slots=20, max_pages=20, page=page, seed=pages)
    for s in range(20):
        p.append([s], [int(p.rng.integers(1, 3 * page))])
    if p.m.error == 0:
        p.fork([3], [19])
    p.free([0, 2, 5, 6, 11])
    p.compact()
    p.same("holes")
    p.compact()
    p.same("none left")
    p.append([0, 2], [page + 1, 3])
    p.same("append behind")
    p.free(list(range(20)))
    p.compact()
    p.same("empty")


def test_more_words_than_threads():
    """Bitmaps of more than 1024 words of 64 pages, with the free pages at the far end."""
    p = Pair(layers=1, pages=66000, hkv=1, slots=3, max_pages=65900, page=16, seed=9)
    p.reserve([0], [65800 * 16])
    p.append([1], [100])
    p.same("far end")
    p.truncate([0], [5 * 16])
    p.compact()
    p.same("compacted")


def test_pages_run_out():
    p = Pair(pages=5, seed=10)
    p.append([0, 1], [33, 16])           # four pages
    p.fork([0], [2])
    p.reserve([2, 1], [1, 1])            # a copy and a page: one too many
    p.same("full")
    assert p.m.error == FULL
    p.write([1], [1])                    # nothing is written, forked, freed or moved
    p.fork([0], [3])
    p.free([0])
    p.compact()
    p.reserve([3], [1])
    p.same("no call does anything")
    with pytest.raises(p.fpx.CacheError) as e:
        p.c.check()
    assert e.value.bits == FULL
    p.m.error = 0
    p.c.check()
    p.append([1], [1])                   # the last page
    p.same("goes on")


def test_a_slot_too_long():
    p = Pair(max_pages=2, seed=11)
    p.append([0, 1], [32, 20])
    p.reserve([1, 0], [1, 1])
    p.same("too long")
    assert p.m.error == TOO_LONG
    with pytest.raises(p.fpx.CacheError):
        p.c.check()
    p.m.error = 0
    p.reserve([1], [2 ** 31 - 1])
    assert p.m.error == TOO_LONG
    p.same("far too long")


def test_write_without_reserve():
    p = Pair(seed=12)
    p.append([0], [20])
    p.fork([0], [1])
    p.write([1], [3])                    # tokens 17 .. 19 lie on a page that slot 0 holds
    p.same("shared")
    assert p.m.error == SHARED
    with pytest.raises(p.fpx.CacheError) as e:
        p.c.check()
    assert e.value.bits == SHARED
    p.m.error = 0
    p.free([1])
    p.write([0], [20])                   # the same tokens again, no longer shared
    p.write([0], [30])                   # more rows than tokens: the first ten are left out
    p.same("own")


@pytest.mark.parametrize("seed", range(6))
def test_a_long_series_of_calls(seed):
    rng = np.random.default_rng(100 + seed)
    page = int(rng.choice([16, 32, 64]))
    p = Pair(pages=150, hkv=1, d=64, slots=10, max_pages=30, page=page, seed=seed)
    for step in range(40):
        op = rng.integers(0, 6)
        slots = rng.permutation(10)[:rng.integers(1, 6)].tolist()
        if op <= 2:
            p.append(slots, rng.integers(0, rng.choice([2, 40, 3 * page]), len(slots)).tolist())
        elif op == 3:
            dst = slots[:max(1, len(slots) // 2)]
            src = [s for s in range(10) if s not in dst]
            p.fork(rng.choice(src, len(dst)).tolist(), dst)
        elif op == 4:
            p.truncate(slots, [int(rng.integers(0, p.m.len[s] + 2)) for s in slots])
        else:
            p.compact()
        p.same(f"seed {seed} step {step} op {op} slots {slots}")
        if p.m.error:
            with pytest.raises(p.fpx.CacheError):
                p.c.check()
            p.m.error = 0


def test_offsets_past_32_bits():
    """A pool of 2^31 elements and more: pages of the last layer lie past 4 GB."""
    import paper_2502_20766_amd as fpx
    layers, pages, hkv, d, page = 2, 9000, 8, 128, 128      # 1.2e9 elements a layer
    c = fpx.Cache(layers, pages, hkv, d, 3, pages, page)
    assert c.k.numel() > 2 ** 31
    fpx.cache_reserve(c, [0], [(pages - 4) * page])          # leaves the last four pages
    g = torch.Generator("cuda").manual_seed(5)
    k = torch.randn(300, hkv, d, generator=g, device="cuda").bfloat16()
    v = torch.randn(300, hkv, d, generator=g, device="cuda").bfloat16()
    fpx.cache_reserve(c, [1], [300])
    fpx.cache_write(c, 1, k, v, [1], [0, 300])
    c.check()
    rows = c.table[1, :3].tolist()
    assert rows == [pages - 4, pages - 3, pages - 2]
    t = torch.arange(300, device="cuda")
    p = c.table[1][t // page].long()
    assert torch.equal(c.k[1][p, :, t % page], k)
    assert torch.equal(c.v[1][p, :, t % page // 16, :, t % 16], v)
    fpx.cache_fork(c, [1], [2])
    fpx.cache_reserve(c, [2], [1])                           # copies page - 2 to page - 1
    assert torch.equal(c.k[1, pages - 1], c.k[1, pages - 2])
    assert torch.equal(c.v[1, pages - 1], c.v[1, pages - 2])
    fpx.cache_free(c, [0])
    fpx.cache_compact(c)
    c.check()
    assert sorted(set(c.table[1, :3].tolist() + c.table[2, :3].tolist())) == [0, 1, 2, 3]
    p = c.table[1][t // page].long()
    assert torch.equal(c.k[1][p, :, t % page], k)
    assert torch.equal(c.v[1][p, :, t % page // 16, :, t % 16], v)


def test_on_another_stream():
    """Every call, workspaces included, on a stream that is not the current one."""
    p, side = Pair(seed=13), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    f = p.fpx
    k = torch.zeros(20, 2, 64, dtype=torch.bfloat16, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    f.cache_init(p.c, stream=side)
    f.cache_reserve(p.c, [0], 20, stream=side)
    for layer in range(2):
        f.cache_write(p.c, layer, k, k, [0], [0, 20], stream=side)
    f.cache_fork(p.c, [0], [1], stream=side)
    f.cache_reserve(p.c, [1], 1, stream=side)
    f.cache_free(p.c, [0], stream=side)
    f.cache_compact(p.c, stream=side)
    side.synchronize()
    zero = np.zeros((20, 2, 64), np.uint16)
    p.m.reserve([0], [20])
    for layer in range(2):
        p.m.write(layer, zero, zero, [0], [0, 20])
    p.m.fork([0], [1])
    p.m.reserve([1], [1])
    p.m.truncate([0], [0])
    p.m.compact()
    p.same()


@pytest.mark.parametrize("bad", ["dtype", "rows", "heads", "inner"])
def test_write_refuses_other_tensors(bad):
    p = Pair(seed=14)
    p.append([0], [4])
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    x = {"dtype": k.float(), "rows": k[:3], "heads": k[:, :1],
         "inner": torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")[..., ::2]}[bad]
    for a, b in ((x, k), (k, x)):
        with pytest.raises(ValueError):
            p.fpx.cache_write(p.c, 0, a, b, [0], [0, 4])
    p.same()
