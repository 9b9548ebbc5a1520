"""Host side of rotations, appends and chunk attention: frequencies, sizes, and the refusal of every bad
argument before any device is touched (these run without a GPU)."""
import ctypes
import os

import numpy as np
import pytest

import paper_2502_20766_amd as fpx
from chunk_model import frequencies

OK, INVALID, UNSUPPORTED, WORKSPACE = (fpx.FP_OK, fpx.FP_ERR_INVALID_ARG, fpx.FP_ERR_UNSUPPORTED,
                                       fpx.FP_ERR_WORKSPACE)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fpx.LIB_PATH):
        from paper_2502_20766_amd import _build
        _build.build()
    return fpx.lib()


def _cache(layers=2, pages=100, hkv=2, d=64, page=64, slots=8, max_pages=10):
    # k, v, meta: addresses that no host-side check dereferences
    return fpx.FpCache(layers, pages, hkv, d, page, slots, max_pages, 4096, 4096, 4096)


def _i32(*x):
    return np.array(x, np.int32)


def _p(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


@pytest.mark.parametrize("rotary", [16, 32, 64, 112, 128])
@pytest.mark.parametrize("kw", [{}, dict(base=500000.0), dict(base=1.0),
                                dict(scaling="linear", factor=4.0),
                                dict(scaling="base", factor=8.0),
                                dict(scaling="parts", factor=8.0, original_len=8192, base=5e5),
                                dict(scaling="parts", factor=8.0, original_len=8192, low_turns=1.0,
                                     high_turns=4.0),
                                dict(scaling="parts", factor=1.0, original_len=100)])
def test_steps_are_fractions_of_a_turn(lib, rotary, kw):
    r = fpx.Rope(rotary, **kw).c
    want = frequencies(rotary, **kw).astype(np.longdouble) / (2 * np.arctan2(np.longdouble(0),
                                                                             np.longdouble(-1)))
    got = np.array(r.step[:rotary // 2], np.uint64).astype(np.longdouble) / np.longdouble(2) ** 64
    # (a double's power is off by some 2^-52 of itself)
    assert np.all(np.abs(got - want) <= 2.0 ** -50 * want + 2.0 ** -64)
    assert r.rotary_dim == rotary and r.amplitude == 1.0


def test_whole_turns_and_negative_frequencies(lib):
    two_pi = 2 * np.pi
    r = fpx.Rope(16, inv_freq=[0.0, two_pi, -two_pi / 4, two_pi * 1.5, 1.0, 1e5, -1.0, 2.0 ** 20]).c
    turn = np.array(r.step[:8], np.uint64) / 2.0 ** 64
    assert turn[0] == 0 and min(turn[1], 1 - turn[1]) < 1e-15 and abs(turn[2] - 0.75) < 1e-15
    assert abs(turn[3] - 0.5) < 1e-15 and abs(turn[4] + turn[6] - 1) < 1e-15


def _params(rotary=64, layout=0, scaling=0, base=1e4, factor=1.0, original=0.0, low=0.0, high=0.0,
            amplitude=1.0, inv_freq=None):
    return fpx.FpRopeParams(rotary, layout, scaling, base, factor, original, low, high, amplitude,
                            None if inv_freq is None else inv_freq.ctypes.data)


INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kw,status", [
    ({}, OK), (dict(rotary=0), INVALID), (dict(rotary=-16), INVALID), (dict(rotary=63), INVALID),
    (dict(rotary=24), UNSUPPORTED), (dict(rotary=144), UNSUPPORTED), (dict(layout=2), INVALID),
    (dict(layout=-1), INVALID), (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID),
    (dict(base=0.0), INVALID), (dict(base=-1.0), INVALID), (dict(base=NAN), INVALID),
    (dict(base=INF), INVALID), (dict(base=1e-9), INVALID),       # a frequency above 2^20
    (dict(scaling=1, factor=0.5), INVALID), (dict(scaling=1, factor=NAN), INVALID),
    (dict(scaling=2, factor=INF), INVALID), (dict(scaling=2, factor=4.0), OK),
    (dict(scaling=3, factor=4.0), INVALID),
    (dict(scaling=3, factor=4.0, original=100.0, low=1.0, high=1.0), INVALID),
    (dict(scaling=3, factor=4.0, original=100.0, low=-1.0, high=1.0), INVALID),
    (dict(scaling=3, factor=4.0, original=NAN, low=1.0, high=2.0), INVALID),
    (dict(scaling=3, factor=4.0, original=100.0, low=1.0, high=2.0), OK),
    (dict(amplitude=NAN), INVALID), (dict(amplitude=INF), INVALID), (dict(amplitude=-1.0), INVALID),
    (dict(amplitude=0.0), OK), (dict(amplitude=1e39), INVALID),
    (dict(inv_freq=np.full(32, 1e-3)), OK), (dict(inv_freq=np.full(32, NAN)), INVALID),
    (dict(inv_freq=np.full(32, 1e7)), INVALID), (dict(inv_freq=np.full(32, -1.0), base=0.0), OK)])
def test_rope_parameters(lib, kw, status):
    p, r = _params(**kw), fpx.FpRope()
    assert lib.fp_rope_init(ctypes.byref(p), ctypes.byref(r)) == status
    assert lib.fp_rope_init(None, ctypes.byref(r)) == INVALID
    assert lib.fp_rope_init(ctypes.byref(p), None) == INVALID


def _rotate(lib, tokens=3, hq=4, hkv=2, d=64, q=4096, qs=256, k=4096, ks=128, pos=4096, rope=True,
            norm=None, qo=4096, qos=256, ko=4096, kos=128):
    r = fpx.Rope(64).ref if rope is True else rope
    return lib.fp_rotate(tokens, hq, hkv, d, q, qs, k, ks, pos, r, norm, qo, qos, ko, kos, None)


@pytest.mark.parametrize("kw,status", [
    (dict(tokens=-1), INVALID), (dict(tokens=(1 << 25) + 1), UNSUPPORTED), (dict(tokens=0), OK),
    (dict(tokens=0, q=None), OK), (dict(hq=0, hkv=0), INVALID), (dict(hq=-1), INVALID),
    (dict(hkv=-1), INVALID), (dict(hq=8193), UNSUPPORTED), (dict(hkv=8193), UNSUPPORTED),
    (dict(d=96), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(q=None), INVALID),
    (dict(q=4104), INVALID), (dict(qs=255), INVALID), (dict(qs=260), INVALID), (dict(qs=248), INVALID),
    (dict(k=None), INVALID), (dict(ko=None), INVALID), (dict(ko=4100), INVALID),
    (dict(kos=120), INVALID), (dict(kos=264), INVALID),      # its own input with another stride
    (dict(qo=4112, qos=250), INVALID), (dict(pos=None), INVALID), (dict(pos=4098), INVALID)])
def test_rotate(lib, kw, status):
    assert _rotate(lib, **kw) == status


def test_rotate_structures(lib):
    wide = fpx.Rope(128)
    assert _rotate(lib, rope=wide.ref) == INVALID             # more than the head has
    for change in (dict(rotary_dim=8), dict(rotary_dim=40), dict(layout=2), dict(amplitude=NAN)):
        r = fpx.Rope(64)
        for name, x in change.items():
            setattr(r.c, name, x)
        assert _rotate(lib, rope=r.ref) == INVALID
    for q, k, f32, eps in ((4104, 4096, 0, 1e-6), (4096, 4097, 0, 1e-6), (4096, 4096, 2, 1e-6),
                           (4096, 4096, 0, 0.0), (4096, 4096, 0, -1.0), (4096, 4096, 1, NAN),
                           (None, None, 0, INF), (None, None, 0, 1e-40)):
        n = fpx.FpHeadNorm(q, k, f32, eps)
        assert _rotate(lib, norm=ctypes.byref(n)) == INVALID


def _append(lib, cache=None, layer=0, slots=_i32(0), cu=_i32(0, 1), hq=4, q=4096, qs=256, k=4096, ks=128,
            v=4096, vs=128, rope=True, norm=None, qo=4096, qos=256):
    r = fpx.Rope(64).ref if rope is True else rope
    n = 1 if slots is None else slots.size
    return lib.fp_cache_append(ctypes.byref(cache or _cache()), layer, n, _p(slots), _p(cu), hq, q, qs,
                               k, ks, v, vs, r, norm, qo, qos, None)


@pytest.mark.parametrize("kw,status", [
    (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(cu=_i32(1, 2)), INVALID),
    (dict(cu=_i32(0, -1)), INVALID), (dict(cu=None), INVALID), (dict(slots=None), INVALID),
    (dict(slots=_i32(8)), INVALID), (dict(slots=_i32(-1)), INVALID),
    (dict(slots=_i32(3, 3), cu=_i32(0, 1, 2)), INVALID),
    (dict(slots=np.zeros(0, np.int32), cu=_i32(0)), INVALID),
    (dict(slots=np.arange(257, dtype=np.int32) % 8, cu=np.arange(258, dtype=np.int32)), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=4104), INVALID), (dict(ks=127), INVALID),
    (dict(vs=132), INVALID), (dict(hq=-1), INVALID), (dict(hq=8193), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(qo=None), INVALID), (dict(qs=248), INVALID), (dict(qos=264), INVALID),
    (dict(qo=4104), INVALID), (dict(cu=_i32(0, 1 << 30)), UNSUPPORTED),
    (dict(cu=_i32(0, 0), k=None, q=None), OK), (dict(rope=fpx.FpRope()), INVALID)])
def test_append(lib, kw, status):
    if isinstance(kw.get("rope"), fpx.FpRope):
        kw = dict(kw, rope=ctypes.byref(kw["rope"]))
    assert _append(lib, **kw) == status


def _batch(slots=(0, 1, -1, 1), cu=(0, 5, 5, 6, 200), hq=4, scale=0.0):
    return fpx.ChunkBatch(slots, cu, hq, scale)


@pytest.mark.parametrize("kw,status", [
    ({}, OK), (dict(slots=(), cu=(0,)), INVALID), (dict(slots=[0] * 257, cu=range(258)), UNSUPPORTED),
    (dict(slots=[-2, 0, 0, 0]), INVALID), (dict(slots=[8, 0, 0, 0]), INVALID),
    (dict(cu=(1, 2, 3, 4, 5)), INVALID), (dict(cu=(0, 3, 2, 4, 5)), INVALID), (dict(hq=3), INVALID),
    (dict(hq=0), INVALID), (dict(hq=16384), UNSUPPORTED), (dict(scale=-1.0), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID),
    (dict(cu=(0, 0, 0, 0, 2 ** 31 - 1)), UNSUPPORTED), (dict(cu=(0, 0, 0, 0, 0)), OK)])
def test_chunk_batch(lib, kw, status):
    c, b, n = _cache(), _batch(**kw), ctypes.c_size_t()
    assert lib.fp_chunk_workspace_size(ctypes.byref(c), b.ref, ctypes.byref(n)) == status
    assert lib.fp_chunk_workspace_size(ctypes.byref(c), b.ref, None) == (status or INVALID)
    if status != OK:
        assert lib.fp_chunk_attn(ctypes.byref(c), b.ref, 0, 4096, 256, 4096, 4096, 1 << 40,
                                 None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(q=None), INVALID),
    (dict(o=None), INVALID), (dict(ws=None), INVALID), (dict(q=4098), INVALID), (dict(o=4104), INVALID),
    (dict(ws=4104), INVALID), (dict(stride=255), INVALID), (dict(stride=260), INVALID),
    (dict(short=1), WORKSPACE)])
def test_chunk_attn(lib, kw, status):
    c, b, n = _cache(), _batch(), ctypes.c_size_t()
    lib.fp_chunk_workspace_size(ctypes.byref(c), b.ref, ctypes.byref(n))
    a = dict(layer=0, q=4096, o=4096, ws=4096, stride=256, short=0)
    a.update(kw)
    assert lib.fp_chunk_attn(ctypes.byref(c), b.ref, a["layer"], a["q"], a["stride"], a["o"], a["ws"],
                             n.value - a["short"], None) == status


def test_chunks_without_a_query_touch_no_device(lib):
    b = _batch(cu=(0, 0, 0, 0, 0))
    assert lib.fp_chunk_attn(ctypes.byref(_cache()), b.ref, 0, None, 256, None, None, 0, None) == OK


def test_binding_refuses_before_the_library():
    for call in (lambda: fpx.Rope(64, layout="pairs"), lambda: fpx.Rope(64, scaling="ntk"),
                 lambda: fpx.Rope(64, inv_freq=[1.0]), lambda: fpx.Rope(64, amplitude=0),
                 lambda: fpx.Rope(16, inv_freq=np.ones(8), scaling="linear"),
                 lambda: fpx.ChunkBatch([0], [0], 4), lambda: fpx.ChunkBatch([0.5], [0, 1], 4),
                 lambda: fpx.rotate(None, None, None, None)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fpx.FlexPrefillError):
        fpx.Rope(40)


@pytest.mark.parametrize("rows,status", [(1 << 24, OK), (1 << 29, UNSUPPORTED)])
def test_chunks_whose_places_no_part_can_count(lib, rows, status):
    """Row tiles times the keys that a slot has room for: up to 2^45 for each of 16 parts."""
    c, n = _cache(), ctypes.c_size_t()
    c.max_pages = (1 << 26) // c.page
    b = _batch(cu=(0, rows, rows, rows, rows))
    assert lib.fp_chunk_workspace_size(ctypes.byref(c), b.ref, ctypes.byref(n)) == status
