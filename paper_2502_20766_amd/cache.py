"""Paged cache of keys and values, and the attention of the next tokens over it.

Marshalling only, as in the rest of the binding: a `Cache` holds the tensors of fp_cache, a
`DecodeBatch` the host arrays of fp_decode with their pointers, and every call enqueues the
library's kernels on `stream`, or on the current stream of the cache's device, without waiting for
the GPU.  All tensors of a call lie on the cache's device; the caller need not have made it current.

    cache = Cache(layers, num_pages, num_kv_heads, head_dim, num_slots, max_pages)
    cache_reserve(cache, [0], [len(prompt)])          # once for all layers
    cache_write(cache, layer, k, v, [0], [0, len(prompt)])    # per layer, beside the prefill
    cache_fork(cache, [0] * 7, range(1, 8))           # eight samples of one prompt
    batch = DecodeBatch(range(8), num_q_heads, group_start=[0, 8], prefix_lens=[len(prompt)])
    # per step: cache_reserve(cache, slots, 1), then per layer cache_write and
    o = decode_attn(q, cache, layer, batch)
    cache_free(cache, slots); cache_compact(cache)
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import (FP_OK, FpCache, FpDecode, _check, _check_tensor, _torch_stream, _workspace, lib)

CACHE_FULL, CACHE_TOO_LONG, CACHE_SHARED, CACHE_SKIPPED = 1, 2, 4, 8
MAX_CACHE_LIST = 256
MAX_QUERIES = 16


class CacheError(RuntimeError):
    """What the device refused (CACHE_* bits), found by Cache.check."""

    def __init__(self, bits: int):
        self.bits = bits
        names = [n for b, n in ((CACHE_FULL, "too few free pages"),
                                (CACHE_TOO_LONG, "a sequence passes max_pages pages"),
                                (CACHE_SHARED, "tokens written without a reserve"),
                                (CACHE_SKIPPED, "later calls and their writes left out"))
                 if bits & b]
        super().__init__("; ".join(names) or f"error bits {bits}")


# These calls are made several times a layer and step, so the host's share of one counts: lists go
# to the library as the bytes of int32 arrays, tensors as plain addresses.

_int32 = np.dtype(np.int32)
_bf16 = _device = _raw_stream = None


def _load_torch():
    """torch's parts that the calls use; importing this package does not load it."""
    global _bf16, _device, _raw_stream
    import torch
    torch.cuda.init()
    _bf16 = torch.bfloat16
    _device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _ints(x, name, n=None):
    """x as an int32 host array of n elements (tobytes and copy make it contiguous)."""
    if (type(x) is np.ndarray and x.dtype is _int32 and x.ndim == 1
            and (n is None or x.size == n)):
        return x
    a = np.ascontiguousarray(x if isinstance(x, np.ndarray) else list(x))
    if a.dtype != np.int32:
        if a.size and not np.issubdtype(a.dtype, np.integer):
            raise ValueError(f"{name} must hold integers")
        if a.size and (a.min() < -2 ** 31 or a.max() >= 2 ** 31):
            raise ValueError(f"{name} must fit 32 bits")
        a = a.astype(np.int32)
    if a.ndim != 1 or (n is not None and a.size != n):
        raise ValueError(f"{name} must be a list of {n if n is not None else 'any number of'} "
                         f"integers, got shape {a.shape}")
    return a


def _check_stream(cache, stream):
    if getattr(stream, "device_index", cache.index) != cache.index:
        raise ValueError(f"the stream is on device {stream.device_index}, the cache on "
                         f"{cache.index}")


def _stream(cache, stream):
    """The raw handle of `stream` or of the current stream of the cache's device."""
    if stream is None:
        return _raw_stream(cache.index)
    _check_stream(cache, stream)
    return stream.cuda_stream


def _there(cache, call, *args):
    """call(*args) with the cache's device current: kernels start on the one that is."""
    import torch
    with torch.cuda.device(cache.index):
        return call(*args)


def _call(status, what):
    if status != FP_OK:
        _check(status, what)


class Cache:
    """A cache and its device tensors: k [layers, num_pages, Hkv, page, d] and v [layers,
    num_pages, Hkv, page / 16, d, 16] in bf16, and the int32 bookkeeping `meta`, of which
    state, used, lens, refs and table are views.  Without k, v and meta they are allocated, and
    the cache is empty; with them the cache is what they hold."""

    def __init__(self, layers, num_pages, num_kv_heads, head_dim, num_slots, max_pages, page=64,
                 device="cuda", k=None, v=None, meta=None):
        import torch
        self.c = FpCache(int(layers), int(num_pages), int(num_kv_heads), int(head_dim),
                         int(page), int(num_slots), int(max_pages), None, None, None)
        n = ctypes.c_size_t()
        _check(lib().fp_cache_meta_size(ctypes.byref(self.c), ctypes.byref(n)),
               "fp_cache_meta_size")
        shape_k = (layers, num_pages, num_kv_heads, page, head_dim)
        shape_v = (layers, num_pages, num_kv_heads, page // 16, head_dim, 16)
        given = [x is not None for x in (k, v, meta)]
        if any(given) and not all(given):
            raise ValueError("k, v and meta come together")
        if not any(given):
            k = torch.empty(shape_k, dtype=torch.bfloat16, device=device)
            v = torch.empty(shape_v, dtype=torch.bfloat16, device=device)
            meta = torch.empty(n.value, dtype=torch.int32, device=device)
        for name, x, shape, dtype in (("k", k, shape_k, torch.bfloat16),
                                      ("v", v, shape_v, torch.bfloat16),
                                      ("meta", meta, (n.value,), torch.int32)):
            _check_tensor(x, name, len(shape), dtype)
            if tuple(x.shape) != tuple(shape):
                raise ValueError(f"{name} has shape {tuple(x.shape)}; the cache needs {shape}")
        self.index = meta.get_device()
        if not k.get_device() == v.get_device() == self.index:
            raise ValueError("k, v and meta must lie on one device")
        if _bf16 is None:
            _load_torch()
        self.k, self.v, self.meta = k, v, meta
        self.heads, self.head_dim = int(num_kv_heads), int(head_dim)
        self.c.k, self.c.v, self.c.meta = k.data_ptr(), v.data_ptr(), meta.data_ptr()
        words = 2 * -(-int(num_pages) // 64)
        sizes = [8, words, int(num_slots), int(num_pages), int(num_slots) * int(max_pages)]
        self.state, self.used, self.lens, self.refs, table = torch.split(meta, sizes)
        self.table = table.view(int(num_slots), int(max_pages))
        self.ref = ctypes.byref(self.c)
        if not any(given):
            cache_init(self)

    def check(self, stream=None):
        """Waits for the calls so far on `stream` or the current stream; if the device refused one
        since the last check, clears the error there, so that calls work again, and raises
        CacheError.  Until then later reserves, forks, truncations and compactions are left out,
        and so are the writes that would follow them.  Calls on other streams are not waited for."""
        if stream is not None:
            _check_stream(self, stream)
            import torch
            with torch.cuda.stream(_torch_stream(stream, self.meta.device)):
                return self.check()
        bits = int(self.state[1].item())
        if bits:
            self.state[1].zero_()
            raise CacheError(bits)


def cache_workspace_size(cache: Cache) -> int:
    """Workspace bytes of cache_reserve and cache_compact."""
    out = ctypes.c_size_t()
    _check(lib().fp_cache_workspace_size(cache.ref, ctypes.byref(out)),
           "fp_cache_workspace_size")
    return out.value


def _given(cache, workspace):
    """The caller's workspace; its size is the library's to check, in bytes."""
    if not (workspace.get_device() == cache.index and workspace.element_size() == 1
            and workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 CUDA tensor on the cache's device")
    return workspace


def _cache_workspace(cache, workspace, stream):
    if workspace is None:
        return _workspace(cache_workspace_size(cache), cache.meta.device, stream)
    return _given(cache, workspace)


def cache_init(cache: Cache, stream=None):
    """Every slot empty, every page free."""
    if _device() != cache.index:
        return _there(cache, cache_init, cache, stream)
    _call(lib().fp_cache_init(cache.ref, _stream(cache, stream)), "fp_cache_init")


def cache_reserve(cache: Cache, slots, counts, workspace=None, stream=None):
    """Room for counts[i] (or the same count for all) more tokens in slots[i], once for all
    layers.  A shared last page that is not full is copied first.  If pages run out or a slot
    would grow past max_pages nothing changes, and Cache.check raises."""
    if _device() != cache.index:
        return _there(cache, cache_reserve, cache, slots, counts, workspace, stream)
    slots = _ints(slots, "slots")
    n = slots.size
    counts = (np.full(n, counts, np.int32) if isinstance(counts, (int, np.integer))
              else _ints(counts, "counts", n))
    ws = _cache_workspace(cache, workspace, stream)
    _call(lib().fp_cache_reserve(cache.ref, n, slots.tobytes(), counts.tobytes(), ws.data_ptr(),
                                 ws.numel(), _stream(cache, stream)), "fp_cache_reserve")


def _check_rows(cache, x, name, heads):
    """Rows, and the stride between them, of a [T, heads, d] bf16 tensor with contiguous rows."""
    shape, stride, d = x.shape, x.stride(), cache.head_dim
    if len(shape) == 3 and x.get_device() == cache.index and x.dtype is _bf16:
        n, h, e = shape
        if h == heads and e == d and (n == 0 or (stride[2] == 1 and (h == 1 or stride[1] == d))):
            return n, stride[0] if n > 1 else heads * d
    raise ValueError(f"{name} must be a bf16 tensor [T, {heads}, {d}] with contiguous rows on the "
                     f"cache's device")


def cache_write(cache: Cache, layer, k, v, slots, cu_seqlens, stream=None):
    """Keys and values of `layer` for the last cu_seqlens[i+1] - cu_seqlens[i] tokens of
    slots[i].  k, v: [T, Hkv, d] bf16, rows contiguous (slices of a fused projection do)."""
    if _device() != cache.index:
        return _there(cache, cache_write, cache, layer, k, v, slots, cu_seqlens, stream)
    slots = _ints(slots, "slots")
    cu = _ints(cu_seqlens, "cu_seqlens", slots.size + 1)
    nk, ks = _check_rows(cache, k, "k", cache.heads)
    nv, vs = _check_rows(cache, v, "v", cache.heads)
    if not nk == nv == cu[-1]:
        raise ValueError(f"k and v have {nk} and {nv} rows; cu_seqlens ends at {cu[-1]}")
    _call(lib().fp_cache_write(cache.ref, layer, slots.size, slots.tobytes(), cu.tobytes(),
                               k.data_ptr(), ks, v.data_ptr(), vs, _stream(cache, stream)),
          "fp_cache_write")


def cache_fork(cache: Cache, src, dst, stream=None):
    """dst[i] becomes a copy of src[i] that shares its pages; what it held is given back."""
    if _device() != cache.index:
        return _there(cache, cache_fork, cache, src, dst, stream)
    src = _ints(src, "src")
    dst = _ints(dst, "dst", src.size)
    _call(lib().fp_cache_fork(cache.ref, src.size, src.tobytes(), dst.tobytes(),
                              _stream(cache, stream)), "fp_cache_fork")


def cache_truncate(cache: Cache, slots, lens, stream=None):
    """slots[i] keeps its first lens[i] tokens (drafts that were not accepted, for one)."""
    if _device() != cache.index:
        return _there(cache, cache_truncate, cache, slots, lens, stream)
    slots = _ints(slots, "slots")
    lens = _ints(lens, "lens", slots.size)
    _call(lib().fp_cache_truncate(cache.ref, slots.size, slots.tobytes(), lens.tobytes(),
                                  _stream(cache, stream)), "fp_cache_truncate")


def cache_free(cache: Cache, slots, stream=None):
    """The slots become empty; their pages are free once no other slot holds them."""
    if _device() != cache.index:
        return _there(cache, cache_free, cache, slots, stream)
    slots = _ints(slots, "slots")
    _call(lib().fp_cache_truncate(cache.ref, slots.size, slots.tobytes(), None,
                                  _stream(cache, stream)), "fp_cache_truncate")


def cache_compact(cache: Cache, workspace=None, stream=None):
    """The pages in use become pages 0 .. state[0]-1, in every layer and table."""
    if _device() != cache.index:
        return _there(cache, cache_compact, cache, workspace, stream)
    ws = _cache_workspace(cache, workspace, stream)
    _call(lib().fp_cache_compact(cache.ref, ws.data_ptr(), ws.numel(), _stream(cache, stream)),
          "fp_cache_compact")


class DecodeBatch:
    """fp_decode and the host arrays that it points to: sequence b is the cache slot slots[b]
    (-1: none) with its last `queries` tokens as queries; sequences group_start[g] ..
    group_start[g+1]-1 begin with the same prefix_lens[g] tokens."""

    def __init__(self, slots, num_q_heads, queries=1, group_start=None, prefix_lens=None,
                 softmax_scale=0.0):
        # copies: the structure keeps their addresses
        self.slots = _ints(slots, "slots").copy()
        self.group_start = self.prefix_lens = None
        if (group_start is None) != (prefix_lens is None):
            raise ValueError("group_start and prefix_lens come together")
        self.c = FpDecode(self.slots.size, self.slots.ctypes.data, int(num_q_heads),
                          int(queries), 0, None, None, float(softmax_scale))
        if group_start is not None:
            self.prefix_lens = _ints(prefix_lens, "prefix_lens").copy()
            self.group_start = _ints(group_start, "group_start",
                                     self.prefix_lens.size + 1).copy()
            self.c.groups = self.prefix_lens.size
            self.c.group_start = self.group_start.ctypes.data
            self.c.prefix_lens = self.prefix_lens.ctypes.data
        self.ref = ctypes.byref(self.c)
        self.rows, self.heads = self.c.batch * self.c.queries, self.c.num_q_heads


def decode_workspace_size(cache: Cache, batch: DecodeBatch) -> int:
    """Workspace bytes of decode_attn."""
    out = ctypes.c_size_t()
    _check(lib().fp_decode_workspace_size(cache.ref, batch.ref, ctypes.byref(out)),
           "fp_decode_workspace_size")
    return out.value


def decode_attn(q, cache: Cache, layer, batch: DecodeBatch, out=None, workspace=None,
                stream=None):
    """Attention of the batch's query tokens over their sequences.  q: [batch * queries, Hq, d]
    bf16, rows contiguous, sequence by sequence; returns o of the same shape.  The last bits of a
    row depend on the rest of the batch; weights over a prefix with more than 32 query rows of a KV
    head are bf16 numbers, others are held to 2^-16 of themselves."""
    if _device() != cache.index:
        return _there(cache, decode_attn, q, cache, layer, batch, out, workspace, stream)
    T, hq, d = batch.rows, batch.heads, cache.head_dim
    n, stride = _check_rows(cache, q, "q", hq)
    if n != T:
        raise ValueError(f"q has {n} rows; the batch has {T} query tokens")
    if out is None:
        out = _workspace(2 * T * hq * d, q.device, stream).view(_bf16).view(T, hq, d)
    else:
        _check_tensor(out, "out", 3)
        if out.get_device() != cache.index:
            raise ValueError("out must lie on the cache's device")
        if out.shape != (T, hq, d):
            raise ValueError(f"out has shape {tuple(out.shape)}; the batch needs {(T, hq, d)}")
    if workspace is None:
        workspace = _workspace(decode_workspace_size(cache, batch), q.device, stream)
    else:
        _given(cache, workspace)
    _call(lib().fp_decode_attn(cache.ref, batch.ref, layer, q.data_ptr(), stride,
                               out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                               _stream(cache, stream)), "fp_decode_attn")
    return out
