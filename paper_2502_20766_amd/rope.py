"""Norms of query and key heads and their rotation by position, before `select` and `sparse_attn`.

Marshalling only, as in the rest of the binding: a `Rope` holds fp_rope, a `HeadNorm` fp_head_norm with
its weights, and a call enqueues one kernel on `stream`, or on the current stream of the tensors'
device, without waiting for the GPU.

    rope = Rope(128, base=500000.0, scaling="parts", factor=8.0, original_len=8192)
    norm = HeadNorm(q_weight, k_weight, eps=1e-6)             # where a model has them
    q, k = rotate(q, k, positions, rope, norm)                # positions: int32 on the GPU, [T]
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import FpHeadNorm, FpRope, FpRopeParams, _check, _workspace, lib
from . import cache as _cache

_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {None: 0, "linear": 1, "base": 2, "parts": 3}


class Rope:
    """How the first `rotary_dim` elements of a head turn with the position: pair i by base^(-2 i /
    rotary_dim) radians per position, or by inv_freq[i].  layout "half": pairs (i, i + rotary_dim /
    2); "interleaved": (2 i, 2 i + 1).  scaling stretches the frequencies by `factor` for contexts
    longer than a model was made for: "linear", all of them; "base", by a larger base; "parts", those
    that make fewer than high_turns turns in original_len positions, those below low_turns wholly, by a
    share that is linear in the turns.  (A share that is linear in the pair's number, between ends that
    are rounded to whole pairs, is another rule, whose angles differ a little: such frequencies are given
    as inv_freq.)  amplitude multiplies cosines and sines."""

    def __init__(self, rotary_dim, base=10000.0, layout="half", scaling=None, factor=1.0,
                 original_len=0, low_turns=1.0, high_turns=32.0, amplitude=1.0, inv_freq=None):
        if layout not in _LAYOUTS or scaling not in _SCALINGS:
            raise ValueError(f"layout is one of {list(_LAYOUTS)}, scaling one of {list(_SCALINGS)}")
        if not amplitude > 0:
            raise ValueError("amplitude must be above zero")
        f = None
        if inv_freq is not None:
            if scaling is not None:
                raise ValueError("inv_freq are the frequencies themselves: scale them before")
            f = np.ascontiguousarray(inv_freq, dtype=np.float64)
            if f.shape != (int(rotary_dim) // 2,):
                raise ValueError(f"inv_freq has shape {f.shape}; rotary_dim {rotary_dim} needs "
                                 f"{(int(rotary_dim) // 2,)}")
        p = FpRopeParams(int(rotary_dim), _LAYOUTS[layout], _SCALINGS[scaling], float(base),
                         float(factor), float(original_len), float(low_turns), float(high_turns),
                         float(amplitude), None if f is None else f.ctypes.data)
        self.c = FpRope()
        _check(lib().fp_rope_init(ctypes.byref(p), ctypes.byref(self.c)), "fp_rope_init")
        self.rotary_dim = int(rotary_dim)
        self.ref = ctypes.byref(self.c)


class HeadNorm:
    """RMS norm of every query and key head: x / sqrt(mean(x^2) + eps) * weight.  Weights: [head_dim]
    on the GPU, bf16 or float32 alike, or None (1)."""

    def __init__(self, q_weight=None, k_weight=None, eps=1e-6):
        import torch
        given = [w for w in (q_weight, k_weight) if w is not None]
        for w in given:
            if not (w.is_cuda and w.dim() == 1 and w.is_contiguous()
                    and w.dtype in (torch.bfloat16, torch.float32)):
                raise ValueError("norm weights must be contiguous bf16 or float32 CUDA tensors of one "
                                 "dim")
        if len(given) == 2 and (given[0].dtype != given[1].dtype
                                or given[0].shape != given[1].shape
                                or given[0].get_device() != given[1].get_device()):
            raise ValueError("norm weights must have one type, size and device")
        self.q_weight, self.k_weight = q_weight, k_weight      # kept: the structure has addresses
        self.dim = given[0].numel() if given else None
        self.index = given[0].get_device() if given else None
        self.c = FpHeadNorm(None if q_weight is None else q_weight.data_ptr(),
                            None if k_weight is None else k_weight.data_ptr(),
                            int(bool(given) and given[0].dtype == torch.float32), float(eps))
        self.ref = ctypes.byref(self.c)


def _refs(rope, norm, d, index):
    """References to the structures of a call on device `index`, None for what it lacks."""
    if norm is None:
        return (None if rope is None else rope.ref), None
    if norm.dim is not None and (norm.dim != d or norm.index != index):
        raise ValueError(f"norm weights of {norm.dim} elements on device {norm.index}; the heads have "
                         f"{d} on {index}")
    return (None if rope is None else rope.ref), norm.ref


def _stride(x, name, shape, index):
    """Elements between tokens of x, a bf16 tensor of `shape` with contiguous rows on device `index`."""
    if x.shape == shape and x.get_device() == index and x.dtype is _cache._bf16:
        n, h, d = shape
        token, head, one = x.stride()
        if n == 0 or (one == 1 and (h == 1 or head == d)):
            return token if n > 1 else h * d
    raise ValueError(f"{name} must be a bf16 tensor of shape {tuple(shape)} with contiguous rows on the "
                     f"device of the others")


def _new(n, h, d, device, stream):
    return _workspace(2 * n * h * d, device, stream)[:2 * n * h * d].view(_cache._bf16).view(n, h, d)


def rotate(q, k, positions, rope, norm=None, q_out=None, k_out=None, stream=None):
    """The heads of q [T, Hq, d] and k [T, Hkv, d] (bf16, rows contiguous, as slices of a fused
    projection have them; one of them may be None), normed where `norm` is given, rotated by
    positions [T] (int32 on the GPU) where `rope` is.  Returns (q_out, k_out), contiguous if not
    given; an output may be its input."""
    first = q if q is not None else k
    if first is None:
        raise ValueError("q or k must be given")
    if _cache._bf16 is None:
        _cache._load_torch()
    index = first.get_device()
    if index < 0:
        raise ValueError("q and k must be CUDA tensors")
    if _cache._device() != index:
        import torch
        with torch.cuda.device(index):
            return rotate(q, k, positions, rope, norm, q_out, k_out, stream)
    if stream is None:
        raw = _cache._raw_stream(index)
    else:
        raw = stream.cuda_stream
        if getattr(stream, "device_index", index) != index:
            raise ValueError(f"the stream is on device {stream.device_index}, the tensors on {index}")
    if len(first.shape) != 3:
        raise ValueError(f"q and k are [T, heads, d], got {tuple(first.shape)}")
    T, heads, d = first.shape
    hq = hkv = qs = ks = qos = kos = 0
    qp = kp = qo = ko = None
    if q is not None:
        hq = heads
        qs = _stride(q, "q", q.shape, index)
        if q_out is None:
            q_out = _new(T, hq, d, q.device, stream)
        qos = _stride(q_out, "q_out", q.shape, index)
        qp, qo = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        hkv = k.shape[1] if len(k.shape) == 3 else 0
        ks = _stride(k, "k", (T, hkv, d), index)
        if k_out is None:
            k_out = _new(T, hkv, d, k.device, stream)
        kos = _stride(k_out, "k_out", (T, hkv, d), index)
        kp, ko = k.data_ptr(), k_out.data_ptr()
    elif k_out is not None:
        raise ValueError("k_out without k")
    at = None
    if rope is not None:
        if not (positions is not None and positions.get_device() == index
                and positions.dtype is _cache._i32 and positions.shape == (T,)
                and (T < 2 or positions.stride(0) == 1)):
            raise ValueError(f"positions must be a contiguous int32 CUDA tensor of {T} elements on the "
                             f"device of the others")
        at = positions.data_ptr()
    r, w = _refs(rope, norm, d, index)
    _cache._call(lib().fp_rotate(T, hq, hkv, d, qp, qs, kp, ks, at, r, w, qo, qos, ko, kos, raw),
                 "fp_rotate")
    return q_out, k_out
