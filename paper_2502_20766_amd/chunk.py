"""Chunks of new tokens: their keys and values appended to a paged cache, normed and rotated on the
way, and their attention over it.

Marshalling only.  A step of a serving loop that takes prompts in chunks, whatever each sequence brings
(one token, a chunk, a whole prompt):

    cu = np.cumsum([0] + counts)
    cache_reserve(cache, slots, counts)                       # once for all layers
    batch = ChunkBatch(slots, cu, num_q_heads)
    # per layer, q, k, v: slices of the layer's fused projection, one row per token
    q = cache_append(cache, layer, q, k, v, slots, cu, rope, norm)
    o = chunk_attn(q, cache, layer, batch)
"""
from __future__ import annotations

import ctypes

from . import FpChunk, _check, _check_tensor, _workspace, lib
from . import cache as _cache
from .cache import Cache, _call, _check_rows, _given, _ints, _stream, _there
from .rope import _new, _refs


def cache_append(cache: Cache, layer, q, k, v, slots, cu_seqlens, rope, norm=None, q_out=None,
                 stream=None):
    """cache_write of keys normed (where `norm` is given) and rotated (where `rope` is) on the way,
    each by its place in its slot, and of values as they are; the queries of the same tokens are normed
    and rotated into q_out, which is returned.  q: [T, Hq, d] or None, k, v: [T, Hkv, d], bf16, rows
    contiguous; q_out may be q.  Tokens beyond a slot's length, and all after a failed reserve, are left
    out, their rows of q_out too; tokens of a page that is not the slot's alone only from the cache."""
    if _cache._device() != cache.index:
        return _there(cache, cache_append, cache, layer, q, k, v, slots, cu_seqlens, rope, norm,
                      q_out, stream)
    slots = _ints(slots, "slots")
    cu = _ints(cu_seqlens, "cu_seqlens", slots.size + 1)
    d = cache.head_dim
    nk, ks = _check_rows(cache, k, "k", cache.heads)
    nv, vs = _check_rows(cache, v, "v", cache.heads)
    if not nk == nv == cu[-1]:
        raise ValueError(f"k and v have {nk} and {nv} rows; cu_seqlens ends at {cu[-1]}")
    hq, qp, qs, qo, qos = 0, None, 0, None, 0
    if q is not None:
        hq = q.shape[1] if len(q.shape) == 3 else 0
        nq, qs = _check_rows(cache, q, "q", hq)
        if q_out is None:
            q_out = _new(nq, hq, d, q.device, stream)
        no, qos = _check_rows(cache, q_out, "q_out", hq)
        if not nq == no == nk or hq < 1:
            raise ValueError(f"q has shape {tuple(q.shape)}, q_out {tuple(q_out.shape)}; the call has "
                             f"{nk} tokens")
        qp, qo = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    r, w = _refs(rope, norm, d, cache.index)
    _call(lib().fp_cache_append(cache.ref, layer, slots.size, slots.tobytes(), cu.tobytes(), hq, qp,
                                qs, k.data_ptr(), ks, v.data_ptr(), vs, r, w, qo, qos,
                                _stream(cache, stream)), "fp_cache_append")
    return q_out


class ChunkBatch:
    """fp_chunk and the host arrays that it points to: rows cu_seqlens[b] .. cu_seqlens[b+1]-1 of q are
    the last tokens of the cache slot slots[b] (-1: none)."""

    def __init__(self, slots, cu_seqlens, num_q_heads, softmax_scale=0.0):
        # copies: the structure keeps their addresses
        self.slots = _ints(slots, "slots").copy()
        self.cu = _ints(cu_seqlens, "cu_seqlens", self.slots.size + 1).copy()
        self.c = FpChunk(self.slots.size, self.slots.ctypes.data, self.cu.ctypes.data,
                         int(num_q_heads), float(softmax_scale))
        self.ref = ctypes.byref(self.c)
        self.rows, self.heads = int(self.cu[-1]), self.c.num_q_heads


def chunk_workspace_size(cache: Cache, batch: ChunkBatch) -> int:
    """Workspace bytes of chunk_attn."""
    out = ctypes.c_size_t()
    _check(lib().fp_chunk_workspace_size(cache.ref, batch.ref, ctypes.byref(out)),
           "fp_chunk_workspace_size")
    return out.value


def chunk_attn(q, cache: Cache, layer, batch: ChunkBatch, out=None, workspace=None, stream=None):
    """Causal attention of the batch's new tokens over their sequences.  q: [T, Hq, d] bf16, rows
    contiguous, sequence by sequence; returns o of the same shape.  Weights are rounded to 2^-8 of
    themselves (decode_attn: 2^-16), and the last bits of a row depend on the rest of the batch."""
    if _cache._device() != cache.index:
        return _there(cache, chunk_attn, q, cache, layer, batch, out, workspace, stream)
    T, hq, d = batch.rows, batch.heads, cache.head_dim
    n, stride = _check_rows(cache, q, "q", hq)
    if n != T:
        raise ValueError(f"q has {n} rows; the batch has {T} query tokens")
    if out is None:
        out = _new(T, hq, d, q.device, stream)
    else:
        _check_tensor(out, "out", 3)
        if out.get_device() != cache.index:
            raise ValueError("out must lie on the cache's device")
        if out.shape != (T, hq, d):
            raise ValueError(f"out has shape {tuple(out.shape)}; the batch needs {(T, hq, d)}")
    if workspace is None:
        workspace = _workspace(chunk_workspace_size(cache, batch), q.device, stream)
    else:
        _given(cache, workspace)
    _call(lib().fp_chunk_attn(cache.ref, batch.ref, layer, q.data_ptr(), stride, out.data_ptr(),
                              workspace.data_ptr(), workspace.numel(), _stream(cache, stream)),
          "fp_chunk_attn")
    return out
