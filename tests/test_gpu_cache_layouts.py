"""Tensors of one KV head or one token, whose strides say nothing where nothing steps along them."""
import numpy as np
import pytest

from cache_model import attend, tolerance
from test_gpu_cache import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _host(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 37])
def test_one_head_of_a_transposed_tensor(d, n):
    import paper_2502_20766_amd as fpx
    g = torch.Generator("cuda").manual_seed(n + d)
    heads = torch.randn(3, 1, n, d, generator=g, device="cuda").bfloat16()    # head by head
    q, k, v = (x.transpose(0, 1) for x in heads)                              # token by token
    assert n == 1 or k.stride(1) != d
    cache = fpx.Cache(1, 4, 1, d, 2, 4, 16)
    fpx.cache_reserve(cache, [1], n)
    fpx.cache_write(cache, 0, k, v, [1], [0, n])
    o = fpx.decode_attn(q[-1:], cache, 0, fpx.DecodeBatch([1], 1))
    cache.check()
    want, mass = attend(_host(q[-1:]), _host(k), _host(v), d ** -0.5)
    assert np.all(np.abs(_host(o) - want) <= tolerance(want, mass))
    if n > 1:                            # several queries: rows d apart
        o = fpx.decode_attn(q[-2:], cache, 0, fpx.DecodeBatch([1], 1, queries=2))
        want, mass = attend(_host(q[-2:]), _host(k), _host(v), d ** -0.5)
        assert np.all(np.abs(_host(o) - want) <= tolerance(want, mass))


def test_several_heads_of_a_transposed_tensor_are_refused():
    import paper_2502_20766_amd as fpx
    cache = fpx.Cache(1, 4, 2, 64, 2, 4, 16)
    fpx.cache_reserve(cache, [1], 5)
    x = torch.zeros(2, 5, 64, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    with pytest.raises(ValueError):
        fpx.cache_write(cache, 0, x, x, [1], [0, 5])
    with pytest.raises(ValueError):
        fpx.decode_attn(x[:1], cache, 0, fpx.DecodeBatch([1], 2))
