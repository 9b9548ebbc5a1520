"""Which device and stream the cache's calls go to, and what they refuse of other devices: with
stand-ins for tensors, streams and the library (these run without a GPU)."""
import contextlib
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2502_20766_amd as fpx  # noqa: E402
from paper_2502_20766_amd import cache as mod  # noqa: E402


class Tensor:
    """What the binding looks at of a contiguous tensor on device `index`."""

    def __init__(self, index, shape=(), dtype=torch.bfloat16):
        self.index, self.shape, self.dtype = index, tuple(shape), dtype
        self.is_cuda, self.device = index >= 0, torch.device("cuda", max(index, 0))

    def get_device(self):
        return self.index

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.dtype.itemsize

    def numel(self):
        return int(np.prod(self.shape))

    def data_ptr(self):
        return 4096

    def view(self, *shape):
        return Tensor(self.index, shape if isinstance(shape[0], int) else self.shape)


class Library:
    """Notes which call came with which stream while which device was current."""

    def __init__(self, gpu):
        self.gpu, self.calls = gpu, []

    def __getattr__(self, name):
        def call(*args):
            if not name.endswith("_size"):
                self.calls.append((name, self.gpu.current, args[-1]))
            return fpx.FP_OK
        return call


@pytest.fixture
def gpu(monkeypatch):
    """Two devices, of which 0 is current; device i's current stream has the handle 1000 + i."""
    g = types.SimpleNamespace(current=0)

    @contextlib.contextmanager
    def device(index):
        before, g.current = g.current, index
        yield
        g.current = before

    g.lib = Library(g)
    monkeypatch.setattr(mod, "lib", lambda: g.lib)
    monkeypatch.setattr(mod, "_bf16", torch.bfloat16)
    monkeypatch.setattr(mod, "_device", lambda: g.current)
    monkeypatch.setattr(mod, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(mod, "_workspace", lambda n, dev, stream: bytes_on(dev.index))
    monkeypatch.setattr(torch.cuda, "device", device)
    return g


def bytes_on(index):
    return Tensor(index, (1 << 20,), torch.uint8)


def cache_on(index):
    c = mod.Cache.__new__(mod.Cache)
    c.c = fpx.FpCache(1, 10, 2, 64, 16, 4, 3, 4096, 4096, 4096)
    c.ref, c.heads, c.head_dim, c.index = None, 2, 64, index
    c.k = c.v = Tensor(index)
    c.meta = Tensor(index, (8,), torch.int32)
    return c


BATCH = fpx.DecodeBatch([0], 4)
CALLS = {
    "fp_cache_init": lambda c, i, **kw: fpx.cache_init(c, **kw),
    "fp_cache_reserve": lambda c, i, **kw: fpx.cache_reserve(c, [0], 1, **kw),
    "fp_cache_write": lambda c, i, **kw: fpx.cache_write(
        c, 0, Tensor(i, (3, 2, 64)), Tensor(i, (3, 2, 64)), [0], [0, 3], **kw),
    "fp_cache_fork": lambda c, i, **kw: fpx.cache_fork(c, [0], [1], **kw),
    "fp_cache_truncate": lambda c, i, **kw: fpx.cache_truncate(c, [0], [1], **kw),
    "fp_cache_compact": lambda c, i, **kw: fpx.cache_compact(c, **kw),
    "fp_decode_attn": lambda c, i, **kw: fpx.decode_attn(Tensor(i, (1, 4, 64)), c, 0, BATCH, **kw),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("index", [0, 1])
def test_calls_go_to_the_cache_s_device(gpu, name, index):
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


def test_check_refuses_a_stream_of_another_device(gpu):
    with pytest.raises(ValueError, match="stream"):
        cache_on(0).check(types.SimpleNamespace(cuda_stream=77, device_index=1))


@pytest.mark.parametrize("other", [1, -1])
def test_tensors_of_another_device_are_refused(gpu, other):
    c, here, there = cache_on(0), Tensor(0, (3, 2, 64)), Tensor(other, (3, 2, 64))
    for k, v in ((here, there), (there, here)):
        with pytest.raises(ValueError):
            fpx.cache_write(c, 0, k, v, [0], [0, 3])
    q = Tensor(0, (1, 4, 64))
    for kw in (dict(out=Tensor(other, (1, 4, 64))), dict(workspace=bytes_on(other))):
        with pytest.raises(ValueError):
            fpx.decode_attn(q, c, 0, BATCH, **kw)
    with pytest.raises(ValueError):
        fpx.decode_attn(Tensor(other, (1, 4, 64)), c, 0, BATCH)
    with pytest.raises(ValueError):
        fpx.cache_reserve(c, [0], 1, workspace=bytes_on(other))
    with pytest.raises(ValueError):
        fpx.cache_compact(c, workspace=bytes_on(other))
    assert gpu.lib.calls == []


@pytest.mark.parametrize("odd", ["k", "v", "meta"])
def test_parts_of_a_cache_lie_on_one_device(odd, monkeypatch):
    monkeypatch.setattr(mod, "_load_torch", lambda: None)
    n = 8 + 2 + 4 + 10 + 12
    parts = {"k": ((1, 10, 2, 16, 64), torch.bfloat16), "v": ((1, 10, 2, 1, 64, 16), torch.bfloat16),
             "meta": ((n,), torch.int32)}
    given = {x: Tensor(1 if x == odd else 0, *y) for x, y in parts.items()}
    with pytest.raises(ValueError, match="device"):
        fpx.Cache(1, 10, 2, 64, 4, 3, 16, **given)
