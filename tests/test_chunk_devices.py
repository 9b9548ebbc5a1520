"""Which device and stream rotate, cache_append and chunk_attn go to, and what they refuse of other
devices: with stand-ins for tensors, streams and the library (these run without a GPU)."""
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2502_20766_amd as fpx  # noqa: E402
from paper_2502_20766_amd import cache as mod  # noqa: E402
from paper_2502_20766_amd import chunk, rope  # noqa: E402
from test_cache_devices import Tensor, bytes_on, cache_on  # noqa: E402
from test_cache_devices import gpu as cache_gpu  # noqa: E402,F401

BATCH = fpx.ChunkBatch([0], [0, 3], 4)
ROPE = object.__new__(rope.Rope)
ROPE.ref = None
CALLS = {
    "fp_rotate": lambda c, i, **kw: fpx.rotate(rows(i, 4), rows(i, 2), at(i), ROPE, **outs(i), **kw),
    "fp_cache_append": lambda c, i, **kw: fpx.cache_append(
        c, 0, rows(i, 4), rows(i, 2), rows(i, 2), [0], [0, 3], ROPE, q_out=rows(i, 4), **kw),
    "fp_chunk_attn": lambda c, i, **kw: fpx.chunk_attn(rows(i, 4), c, 0, BATCH, out=rows(i, 4), **kw),
}


def rows(index, heads):
    return Tensor(index, (3, heads, 64))


def at(index):
    return Positions(index, (3,), torch.int32)


def outs(index):
    return dict(q_out=rows(index, 4), k_out=rows(index, 2))


class Positions(Tensor):
    def stride(self, dim=None):
        return (1,) if dim is None else 1


@pytest.fixture
def gpu(cache_gpu, monkeypatch):     # noqa: F811
    for m in (rope, chunk):
        monkeypatch.setattr(m, "lib", lambda: cache_gpu.lib)
    monkeypatch.setattr(mod, "_i32", torch.int32)
    monkeypatch.setattr(chunk, "_workspace", lambda n, dev, stream: bytes_on(dev.index))
    return cache_gpu


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("index", [0, 1])
def test_calls_go_to_the_device_of_their_tensors(gpu, name, index):
    CALLS[name](cache_on(index), index)
    assert gpu.lib.calls == [(name, index, 1000 + index)] and gpu.current == 0


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_a_given_stream(gpu, name):
    stream = types.SimpleNamespace(cuda_stream=77, device_index=1)
    CALLS[name](cache_on(1), 1, stream=stream)
    CALLS[name](cache_on(1), 1, stream=types.SimpleNamespace(cuda_stream=78))    # a handle alone
    assert gpu.lib.calls == [(name, 1, 77), (name, 1, 78)]
    with pytest.raises(ValueError, match="stream"):
        CALLS[name](cache_on(0), 0, stream=stream)
    assert len(gpu.lib.calls) == 2


@pytest.mark.parametrize("other", [1, -1])
def test_tensors_of_another_device_are_refused(gpu, other):
    c, good = cache_on(0), dict(q=rows(0, 4), k=rows(0, 2), positions=at(0), **outs(0))
    for name in good:
        if name == "q":
            continue                             # (the call is on q's device)
        bad = dict(good)
        bad[name] = type(good[name])(other, good[name].shape, good[name].dtype)
        with pytest.raises(ValueError):
            fpx.rotate(bad["q"], bad["k"], bad["positions"], ROPE, None, bad["q_out"], bad["k_out"])
    with pytest.raises(ValueError):
        fpx.rotate(rows(-1, 4), None, at(0), ROPE)
    norm = object.__new__(rope.HeadNorm)
    norm.ref, norm.dim, norm.index = None, 64, other
    with pytest.raises(ValueError, match="norm"):
        fpx.rotate(good["q"], good["k"], good["positions"], ROPE, norm, **outs(0))
    with pytest.raises(ValueError, match="norm"):
        fpx.cache_append(c, 0, rows(0, 4), rows(0, 2), rows(0, 2), [0], [0, 3], ROPE, norm,
                         q_out=rows(0, 4))
    for odd in range(4):
        i = [other if j == odd else 0 for j in range(4)]
        with pytest.raises(ValueError):
            fpx.cache_append(c, 0, rows(i[0], 4), rows(i[1], 2), rows(i[2], 2), [0], [0, 3], ROPE,
                             q_out=rows(i[3], 4))
    for kw in (dict(out=rows(other, 4)), dict(out=rows(0, 4), workspace=bytes_on(other))):
        with pytest.raises(ValueError):
            fpx.chunk_attn(rows(0, 4), c, 0, BATCH, **kw)
    with pytest.raises(ValueError):
        fpx.chunk_attn(rows(other, 4), c, 0, BATCH, out=rows(0, 4))
    assert gpu.lib.calls == []
