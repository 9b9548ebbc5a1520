"""cache_append where a page of a slot is not the slot's alone: its keys and values are left out, the queries
of the same tokens are not."""
import numpy as np
import pytest

from cache_model import bits
from test_gpu_append import Append, _bits
from test_gpu_cache import gpu  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("d,hq", [(64, 4), (128, 9)])
def test_queries_of_shared_pages(d, hq):
    a = Append(hq, norm=True, layers=1, pages=8, hkv=2, d=d, slots=3, max_pages=4, page=16, seed=d)
    a.append([0, 1], [20, 7])
    a.fork([0], [2])
    before = _bits(a.c.k), _bits(a.c.v)
    x = a._dev(bits(a.rng.standard_normal((5, hq + 4, d))))
    # (neither slot has been given room, and slot 0 shares its pages)
    q = a.fpx.cache_append(a.c, 0, x[:, :hq], x[:, hq:hq + 2], x[:, hq + 2:], [0, 1], [0, 3, 5], a.rope,
                           a.norm)
    at = torch.tensor([17, 18, 19, 5, 6], dtype=torch.int32, device="cuda")
    want, keys = a.fpx.rotate(x[:, :hq], x[:, hq:hq + 2], at, a.rope, a.norm)
    assert torch.equal(q, want)
    k, v = _bits(a.c.k), _bits(a.c.v)
    own = int(a.m.rows[1][0])                 # slot 1's page takes its two tokens
    assert np.array_equal(k[0, own, :, 5:7], _bits(keys[3:]).transpose(1, 0, 2))
    k[0, own, :, 5:7], v[0, own, :, 0, :, 5:7] = before[0][0, own, :, 5:7], before[1][0, own, :, 0, :, 5:7]
    assert np.array_equal(k, before[0]) and np.array_equal(v, before[1])
    with pytest.raises(a.fpx.CacheError) as e:
        a.c.check()
    assert e.value.bits == a.fpx.CACHE_SHARED
