"""Host side of the cache calls: workspaces that the kernels' int32 lists do not fit (these run
without a GPU)."""
import ctypes

import pytest

import paper_2502_20766_amd as fpx
from test_cache_abi import INVALID, WORKSPACE, _cache, _i32, _p, lib  # noqa: F401


@pytest.mark.parametrize("off", [1, 2, 3])
def test_workspaces_hold_int32_lists(lib, off):  # noqa: F811
    c, s = ctypes.byref(_cache()), _i32(0)
    at = ctypes.c_void_p(4096 + off)
    assert lib.fp_cache_reserve(c, 1, _p(s), _p(s), at, 1 << 20, None) == INVALID
    assert lib.fp_cache_compact(c, at, 1 << 20, None) == INVALID


def test_workspaces_at_any_int32(lib):  # noqa: F811
    """At multiples of four the size is looked at as before."""
    c, s = ctypes.byref(_cache()), _i32(0)
    for off in (4, 8, 12):
        at = ctypes.c_void_p(4096 + off)
        assert lib.fp_cache_reserve(c, 1, _p(s), _p(s), at, 16, None) == WORKSPACE
        assert lib.fp_cache_compact(c, at, 16, None) == WORKSPACE
