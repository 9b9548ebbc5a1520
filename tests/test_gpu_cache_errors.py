"""What the cache does between an error on the device and the check that finds it: tokens that are
there already stay, whichever call was left out."""
import pytest

from cache_model import TOO_LONG
from test_gpu_cache import Pair, gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _shared(seed):
    """Three sequences, of which slot 1 has written onto a page that slot 0 holds too."""
    p = Pair(seed=seed)
    p.append([0, 2], [20, 37])
    p.fork([0], [1])
    p.write([1], [3])
    p.same("shared")
    return p


LEFT_OUT = {
    # a step of another sequence, a shorter one, drafts taken back, a copy
    "reserve": lambda p: p.fpx.cache_reserve(p.c, [2], [3]),
    "truncate": lambda p: p.fpx.cache_truncate(p.c, [2], [30]),
    "fork": lambda p: p.fpx.cache_fork(p.c, [0], [2]),
}


@pytest.mark.parametrize("call", sorted(LEFT_OUT))
def test_no_token_is_overwritten_after_a_call_that_was_left_out(call):
    p = _shared(30)
    before = [x.clone() for x in (p.c.meta, p.c.k, p.c.v)]
    x = torch.randn(3, 2, 64, device="cuda").bfloat16()
    for _ in range(2):                   # two steps before the next check
        LEFT_OUT[call](p)
        for layer in range(2):
            p.fpx.cache_write(p.c, layer, x, x, [2], [0, 3])
    same = p.c.meta == before[0]
    same[1] = True                       # the error bits
    assert bool(same.all())
    for a, b in zip((p.c.k, p.c.v), before[1:]):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    with pytest.raises(p.fpx.CacheError) as e:
        p.c.check()
    assert e.value.bits == p.fpx.CACHE_SHARED | p.fpx.CACHE_SKIPPED
    assert "left out" in str(e.value)
    p.m.error = 0
    p.c.check()
    p.append([2, 0], [3, 1])             # slot 0 takes a copy of the page that it shares
    p.same("goes on")


def test_the_step_that_sets_the_bit_writes_its_other_layers():
    """Only what is not the slot's alone is left out of a step whose reserve was made."""
    p = Pair(seed=31)
    p.append([0], [20])
    p.fork([0], [1])
    p.reserve([2], [5])
    p.write([1, 2], [3, 5])              # slot 1 without a reserve, slot 2 with one
    p.same("other slot written in both layers")
    with pytest.raises(p.fpx.CacheError) as e:
        p.c.check()
    assert e.value.bits == p.fpx.CACHE_SHARED


def test_compaction_that_is_left_out_stops_no_write():
    """It would not have changed a length, so a write still finds its place."""
    p = _shared(32)
    p.compact()
    p.write([2], [3])
    p.same("written")
    with pytest.raises(p.fpx.CacheError) as e:
        p.c.check()
    assert e.value.bits == p.fpx.CACHE_SHARED


@pytest.mark.parametrize("handle", ["stream", "raw"])
def test_check_of_calls_on_another_stream(handle):
    """The error of a call that is still waiting on its stream is found there, and cleared there."""
    p, side = Pair(seed=33), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    given = side

    class Raw:                           # a stream of another library: its handle alone
        cuda_stream = side.cuda_stream

    if handle == "raw":
        given = Raw()
    for _ in range(2):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        p.fpx.cache_reserve(p.c, [0], [10 ** 6], stream=given)
        with pytest.raises(p.fpx.CacheError) as e:
            p.c.check(stream=given)
        assert e.value.bits == TOO_LONG
        p.c.check(stream=given)
    p.append([0], [5])
    p.same()
