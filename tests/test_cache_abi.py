"""Host side of the cache and decoding calls: sizes, and the refusal of every bad argument before
any device is touched (these run without a GPU)."""
import ctypes
import os

import numpy as np
import pytest

import paper_2502_20766_amd as fpx

INVALID, UNSUPPORTED, WORKSPACE = (fpx.FP_ERR_INVALID_ARG, fpx.FP_ERR_UNSUPPORTED,
                                   fpx.FP_ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fpx.LIB_PATH):
        from paper_2502_20766_amd import _build
        _build.build()
    return fpx.lib()


def _cache(layers=2, pages=100, hkv=2, d=64, page=64, slots=8, max_pages=10, k=4096, v=4096,
           meta=4096):
    # k, v, meta: addresses that no host-side check dereferences
    return fpx.FpCache(layers, pages, hkv, d, page, slots, max_pages, k, v, meta)


def _i32(*x):
    return np.array(x, np.int32)


def _p(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


@pytest.mark.parametrize("kw,status", [
    ({}, fpx.FP_OK),
    (dict(page=16), fpx.FP_OK),
    (dict(page=256, d=128), fpx.FP_OK),
    (dict(page=8), UNSUPPORTED),
    (dict(page=48), UNSUPPORTED),
    (dict(page=512), UNSUPPORTED),
    (dict(d=96), UNSUPPORTED),
    (dict(d=0), INVALID),
    (dict(layers=0), INVALID),
    (dict(pages=0), INVALID),
    (dict(pages=(1 << 22) + 1), UNSUPPORTED),
    (dict(hkv=0), INVALID),
    (dict(hkv=1025), UNSUPPORTED),
    (dict(slots=0), INVALID),
    (dict(slots=65537), UNSUPPORTED),
    (dict(max_pages=0), INVALID),
    (dict(max_pages=(1 << 20) + 1), UNSUPPORTED),            # over 2^26 tokens
    (dict(max_pages=1 << 20, slots=2048), UNSUPPORTED),      # table of 2^31 entries
])
def test_cache_sizes(lib, kw, status):
    c, n = _cache(**kw), ctypes.c_size_t()
    assert lib.fp_cache_meta_size(ctypes.byref(c), ctypes.byref(n)) == status
    assert lib.fp_cache_workspace_size(ctypes.byref(c), ctypes.byref(n)) == status
    if status == fpx.FP_OK:
        assert n.value >= 12 * c.num_pages and n.value % 256 == 0
        lib.fp_cache_meta_size(ctypes.byref(c), ctypes.byref(n))
        assert n.value == (8 + 2 * -(-c.num_pages // 64) + c.num_slots + c.num_pages
                           + c.num_slots * c.max_pages)
    assert lib.fp_cache_meta_size(None, ctypes.byref(n)) == INVALID
    assert lib.fp_cache_init(ctypes.byref(_cache(**dict(kw, k=None))), None) != fpx.FP_OK


@pytest.mark.parametrize("kw", [dict(k=None), dict(v=None), dict(meta=None), dict(k=4104),
                                dict(v=4098), dict(meta=4100)])
def test_pointers(lib, kw):
    c, ws = ctypes.byref(_cache(**kw)), ctypes.c_void_p(4096)
    s, n = _i32(0), _i32(1)
    assert lib.fp_cache_init(c, None) == INVALID
    assert lib.fp_cache_reserve(c, 1, _p(s), _p(n), ws, 1 << 20, None) == INVALID
    assert lib.fp_cache_fork(c, 1, _p(s), _p(n), None) == INVALID
    assert lib.fp_cache_truncate(c, 1, _p(s), None, None) == INVALID
    assert lib.fp_cache_compact(c, ws, 1 << 20, None) == INVALID
    assert lib.fp_cache_write(c, 0, 1, _p(s), _p(_i32(0, 1)), 4096, 128, 4096, 128,
                              None) == INVALID


@pytest.mark.parametrize("slots,status", [
    (None, INVALID), (_i32(-1), INVALID), (_i32(8), INVALID), (_i32(3, 3), INVALID),
    (np.zeros(0, np.int32), INVALID), (np.zeros(257, np.int32), UNSUPPORTED)])
def test_slot_lists(lib, slots, status):
    c, ws = ctypes.byref(_cache()), ctypes.c_void_p(4096)
    n = 1 if slots is None else slots.size
    ones = np.ones(max(n, 1), np.int32)
    assert lib.fp_cache_reserve(c, n, _p(slots), _p(ones), ws, 1 << 20, None) == status
    assert lib.fp_cache_truncate(c, n, _p(slots), None, None) == status
    assert lib.fp_cache_fork(c, n, _p(ones), _p(slots), None) == status
    cu = np.arange(max(n, 1) + 1, dtype=np.int32)
    assert lib.fp_cache_write(c, 0, n, _p(slots), _p(cu), 4096, 128, 4096, 128, None) == status


def test_reserve_truncate_fork_compact(lib):
    c, ws = ctypes.byref(_cache()), ctypes.c_void_p(4096)
    s = _i32(0, 1)
    need = ctypes.c_size_t()
    lib.fp_cache_workspace_size(c, ctypes.byref(need))
    assert lib.fp_cache_reserve(c, 2, _p(s), _p(_i32(1, -1)), ws, 1 << 20, None) == INVALID
    assert lib.fp_cache_reserve(c, 2, _p(s), None, ws, 1 << 20, None) == INVALID
    assert lib.fp_cache_reserve(c, 2, _p(s), _p(_i32(1, 1)), None, 1 << 20, None) == INVALID
    assert lib.fp_cache_reserve(c, 2, _p(s), _p(_i32(1, 1)), ws, need.value - 1,
                                None) == WORKSPACE
    assert lib.fp_cache_truncate(c, 2, _p(s), _p(_i32(0, -1)), None) == INVALID
    assert lib.fp_cache_compact(c, None, 1 << 20, None) == INVALID
    assert lib.fp_cache_compact(c, ws, need.value - 1, None) == WORKSPACE
    assert lib.fp_cache_fork(c, 2, _p(_i32(4, 1)), _p(_i32(1, 2)), None) == INVALID  # src in dst
    assert lib.fp_cache_fork(c, 2, _p(_i32(4, 4)), _p(_i32(2, 2)), None) == INVALID
    assert lib.fp_cache_fork(c, 2, _p(_i32(4, 9)), _p(_i32(1, 2)), None) == INVALID
    assert lib.fp_cache_fork(c, 2, None, _p(_i32(1, 2)), None) == INVALID


@pytest.mark.parametrize("kw", [
    dict(layer=-1), dict(layer=2), dict(cu=_i32(1, 2)), dict(cu=_i32(0, -1)), dict(cu=None),
    dict(k=None), dict(v=None), dict(k=4104), dict(v=4104), dict(ks=127), dict(vs=120),
    dict(ks=132), dict(vs=129)])
def test_write(lib, kw):
    a = dict(layer=0, cu=_i32(0, 1), k=4096, v=4096, ks=128, vs=128)
    a.update(kw)
    assert lib.fp_cache_write(ctypes.byref(_cache()), a["layer"], 1, _p(_i32(0)), _p(a["cu"]),
                              a["k"], a["ks"], a["v"], a["vs"], None) == INVALID


def test_write_of_nothing_touches_no_device(lib):
    assert lib.fp_cache_write(ctypes.byref(_cache()), 0, 2, _p(_i32(0, 1)), _p(_i32(0, 0, 0)),
                              None, 128, None, 128, None) == fpx.FP_OK


def test_write_of_too_much(lib):
    """More (64 tokens, KV head) pieces than one launch takes."""
    cu = _i32(0, 1 << 30)
    assert lib.fp_cache_write(ctypes.byref(_cache()), 0, 1, _p(_i32(0)), _p(cu), 4096, 128, 4096,
                              128, None) == UNSUPPORTED


def _batch(slots=(0, 1, -1, 1), hq=4, queries=1, start=None, prefix=None, scale=0.0):
    return fpx.DecodeBatch(slots, hq, queries, start, prefix, scale)


@pytest.mark.parametrize("kw,status", [
    ({}, fpx.FP_OK),
    (dict(queries=16), fpx.FP_OK),
    (dict(start=[0, 2, 4], prefix=[64, 0]), fpx.FP_OK),
    (dict(slots=()), INVALID),
    (dict(slots=[0] * 257), UNSUPPORTED),
    (dict(slots=[-2]), INVALID),
    (dict(slots=[8]), INVALID),
    (dict(hq=3), INVALID),
    (dict(hq=0), INVALID),
    (dict(hq=16384), UNSUPPORTED),
    (dict(queries=0), INVALID),
    (dict(queries=17), UNSUPPORTED),
    (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID),
    (dict(start=[0, 2, 3], prefix=[1, 1]), INVALID),
    (dict(start=[1, 2, 4], prefix=[1, 1]), INVALID),
    (dict(start=[0, 4, 4], prefix=[1, 1]), INVALID),
    (dict(start=[0, 5, 4], prefix=[1, 1]), INVALID),
    (dict(start=[0, 2, 4], prefix=[1, -1]), INVALID),
    (dict(start=[0, 1, 2, 3, 4, 4], prefix=[1] * 5), INVALID),
])
def test_decode_batch(lib, kw, status):
    c, b, n = _cache(), _batch(**kw), ctypes.c_size_t()
    assert lib.fp_decode_workspace_size(ctypes.byref(c), b.ref, ctypes.byref(n)) == status
    if status != fpx.FP_OK:
        assert lib.fp_decode_attn(ctypes.byref(c), b.ref, 0, 4096, 1 << 20, 4096, 4096, 1 << 40,
                                  None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(q=None), INVALID),
    (dict(o=None), INVALID), (dict(ws=None), INVALID), (dict(q=4098), INVALID),
    (dict(stride=255), INVALID), (dict(stride=260), INVALID), (dict(short=1), WORKSPACE)])
def test_decode_attn(lib, kw, status):
    c, b, n = _cache(), _batch(), ctypes.c_size_t()
    lib.fp_decode_workspace_size(ctypes.byref(c), b.ref, ctypes.byref(n))
    a = dict(layer=0, q=4096, o=4096, ws=4096, stride=256, short=0)
    a.update(kw)
    assert lib.fp_decode_attn(ctypes.byref(c), b.ref, a["layer"], a["q"], a["stride"], a["o"],
                              a["ws"], n.value - a["short"], None) == status


def test_line_too_long(lib):
    """2^20 tiles a sequence, 1024 KV heads: more tiles than a 32-bit line holds."""
    c = _cache(hkv=1024, d=64, page=64, max_pages=1 << 20, slots=4)
    b, n = fpx.DecodeBatch([0, 1, 2], 1024), ctypes.c_size_t()
    assert lib.fp_decode_workspace_size(ctypes.byref(c), b.ref,
                                        ctypes.byref(n)) == UNSUPPORTED


def test_binding_refuses_before_the_library():
    with pytest.raises(ValueError):
        fpx.DecodeBatch([0], 4, group_start=[0, 1])
    with pytest.raises(ValueError):
        fpx.DecodeBatch([0], 4, group_start=[0, 1, 2], prefix_lens=[3])
    with pytest.raises(ValueError):
        fpx.DecodeBatch([0.5], 4)
    with pytest.raises(ValueError):
        fpx.DecodeBatch([2 ** 31], 4)
    with pytest.raises(fpx.FlexPrefillError):
        fpx.Cache(1, 10, 2, 96, 2, 4, device="cpu")
    assert "free pages" in str(fpx.CacheError(fpx.CACHE_FULL))
