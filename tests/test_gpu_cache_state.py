"""Compaction of bookkeeping that does not agree with itself, as a caller's own `meta` may: nothing
moves, and nothing is read or written outside of the cache."""
import pytest

from test_gpu_cache import Pair, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("pages", [60, 64, 130])
@pytest.mark.parametrize("change", ["more in use", "fewer in use", "bits past the last page"])
def test_compaction_of_a_state_that_does_not_fit(pages, change):
    p = Pair(pages=pages, slots=6, seed=pages)
    p.append([0, 1, 2], [40, 50, 60])    # three, four and four pages
    p.free([1])                          # four holes, all below the seven pages in use
    if change == "more in use":          # more holes than pages to fill them
        p.c.state[0] += 6
    elif change == "fewer in use":       # more pages than holes
        p.c.state[0] -= 3
    elif pages % 64:
        p.c.used[-1] |= -(2 ** 31)
    before = [x.clone() for x in (p.c.meta, p.c.k, p.c.v)]
    # what an earlier call left in the workspace is no page of this cache
    n = p.fpx.cache_workspace_size(p.c)
    ws = torch.full((4 * n,), 0x7B, dtype=torch.uint8, device="cuda")
    p.fpx.cache_compact(p.c, workspace=ws[:n])
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0x7B).all())
    if change == "bits past the last page":
        # (the bit is none of a page; the others are as many as the holes)
        p.c.used[-1] &= 2 ** 31 - 1
        p.compact()
        p.same()
        return
    for a, b in zip((p.c.meta, p.c.k, p.c.v), before):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
