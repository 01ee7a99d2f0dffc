"""Binding of the serving entry points: exact attention over packed prompts, and a paged cache that holds keys and values in
4 bits, with its scheduling.  Argument marshalling only, like `binding.py`; lengths, tables and slots are int32 CUDA tensors
that only the kernels read, so nothing here waits for the GPU.

A cache is a uint8 tensor [pages, kv_heads, page_tokens / 16, 20 d] (`cache_pages` makes one; include/hyperattn.h has the order of
its bytes).  A decode step of a server:

    plan = cache_plan(lengths, new, table, free, n_free, page_tokens, rows)       # pages, slots and positions of the step's tokens
    cache_store(cache, k, v, plan.slots)                                          # for every layer: the new keys and values,
    out, lse = cache_attention(q, cache, plan.table, plan.lengths)                # attention over all that is cached
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

import torch

from .binding import BF16, FP32, HyperAttnError, _call, _raw_stream, lib

FP16 = 2
_CODES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
PLAN_MAX_REQUESTS = 4096


class _Cache(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("num_pages", C.c_int), ("page_tokens", C.c_int), ("kv_heads", C.c_int), ("d", C.c_int)]


class _Plan(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("lengths", "new_tokens", "table", "free_pages", "n_free")]
                + [(n, C.c_int) for n in ("requests", "table_width", "num_free", "page_tokens", "rows")]
                + [(n, C.c_void_p) for n in ("slots", "positions", "cu_new", "cu_lengths", "lengths_out", "table_out", "free_out",
                                             "n_free_out", "stream")])


class _CacheAttention(C.Structure):
    _fields_ = [("cache", _Cache), ("q", C.c_void_p), ("q_row_stride", C.c_longlong), ("q_head_stride", C.c_longlong),
                ("out", C.c_void_p), ("lse", C.c_void_p), ("table", C.c_void_p), ("lengths", C.c_void_p),
                ("requests", C.c_int), ("table_width", C.c_int), ("q_heads", C.c_int), ("dtype", C.c_int), ("out_dtype", C.c_int),
                ("softmax_scale", C.c_float), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class _Prompt(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v")]
                + [(n, C.c_longlong) for n in ("q_row_stride", "q_head_stride", "k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")]
                + [(n, C.c_void_p) for n in ("out", "lse", "cu_q", "cu_k")]
                + [(n, C.c_int) for n in ("requests", "q_rows", "k_rows", "q_heads", "kv_heads", "d", "causal", "dtype", "out_dtype")]
                + [("softmax_scale", C.c_float), ("stream", C.c_void_p)])


_typed = False


def _lib():
    global _typed
    L = lib()
    if not _typed:
        i, p, ll = C.c_int, C.c_void_p, C.c_longlong
        for name, args in (("hyperattn_cache_plan", [C.POINTER(_Plan)]),
                           ("hyperattn_cache_store", [C.POINTER(_Cache), p, p, i, i, ll, ll, ll, ll, p, p]),
                           ("hyperattn_cache_read", [C.POINTER(_Cache), p, i, i, p, p, i, p, p, i, p]),
                           ("hyperattn_cache_attention", [C.POINTER(_CacheAttention)]),
                           ("hyperattn_cache_attention_workspace_bytes", [C.POINTER(_CacheAttention), C.POINTER(C.c_size_t)]),
                           ("hyperattn_prompt_attention", [C.POINTER(_Prompt)])):
            getattr(L, name).restype = i
            getattr(L, name).argtypes = args
        _typed = True
    return L


def _ints(device, **tensors):
    """The int32 tensors of a call: on its device, contiguous."""
    for name, t in tensors.items():
        if t.dtype != torch.int32 or t.device != device or not t.is_contiguous():
            raise HyperAttnError(f"{name} must be a contiguous int32 tensor on {device}")


def _rows(x):
    """x [rows, heads, d] with strides that the kernels take: d contiguous, the others and the address in steps of 16 bytes."""
    s = x.stride()
    if s[2] != 1 or s[0] % 8 or s[1] % 8 or s[0] <= 0 or s[1] <= 0 or x.data_ptr() % 16:
        return x.clone(memory_format=torch.contiguous_format)
    return x


def _code(t, what):
    code = _CODES.get(t)
    if code is None:
        raise HyperAttnError(f"unsupported dtype {t} of {what}")
    return code


def _cache_of(cache):
    if not cache.is_cuda or cache.dtype != torch.uint8 or cache.dim() != 4 or not cache.is_contiguous() or cache.shape[3] not in (1280, 2560):
        raise HyperAttnError("a cache is a contiguous CUDA uint8 tensor [pages, kv_heads, page_tokens / 16, 20 d], d 64 or 128")
    pages, heads, blocks, size = cache.shape
    return _Cache(cache.data_ptr(), pages, blocks * 16, heads, size // 20)


def cache_pages(pages, kv_heads, d, page_tokens=64, device="cuda"):
    """An empty cache of `pages` pages of `page_tokens` tokens (a multiple of 16) for one layer."""
    if d not in (64, 128) or page_tokens <= 0 or page_tokens % 16 or page_tokens > 1024 or pages <= 0 or kv_heads <= 0:
        raise HyperAttnError("d must be 64 or 128, page_tokens a multiple of 16 up to 1024")
    return torch.zeros(pages, kv_heads, page_tokens // 16, 20 * d, dtype=torch.uint8, device=device)


class CachePlan(NamedTuple):
    slots: torch.Tensor       # [rows] slot of every new token, -1: none
    positions: torch.Tensor   # [rows] its position in its request, -1: none
    cu_new: torch.Tensor      # [requests + 1] first row of every request's new tokens
    cu_len: torch.Tensor      # [requests + 1] running sum of `lengths`
    lengths: torch.Tensor     # [requests] tokens in the cache after the step
    table: torch.Tensor       # [requests, width] pages of every request, -1: none
    free: torch.Tensor        # the stack of free pages, -1: none
    n_free: torch.Tensor      # [1] entries on it


def cache_plan(lengths, new, table, free, n_free, page_tokens, rows, stream=None):
    """One scheduling step: hands pages to the requests' new tokens, takes back those of ended requests (new < 0), and says where
    every token of the packed batch of `rows` rows goes.  lengths, new [requests], table [requests, width], free [any], n_free [1]:
    int32 CUDA tensors, not changed.  Requests whose pages cannot be had keep their length and get no slots.  Returns a CachePlan."""
    if not lengths.is_cuda:
        raise HyperAttnError("lengths must be a CUDA tensor (there is no CPU path)")
    dev = lengths.device
    _ints(dev, lengths=lengths, new=new, table=table, free=free, n_free=n_free)
    R = lengths.shape[0]
    if lengths.dim() != 1 or new.shape != lengths.shape or table.dim() != 2 or table.shape[0] != R or free.dim() != 1 or n_free.numel() != 1:
        raise HyperAttnError("lengths and new are [requests], table [requests, width], free [pages], n_free [1]")
    if R == 0:
        none = torch.full((2, rows), -1, dtype=torch.int32, device=dev)
        zero = torch.zeros(2, 1, dtype=torch.int32, device=dev)
        return CachePlan(none[0], none[1], zero[0], zero[1], lengths.clone(), table.clone(), free.clone(), n_free.clone())
    W, F = table.shape[1], free.shape[0]
    new_ints = lengths.new_empty
    # one allocation for the small results
    both = new_ints(2 * rows + 3 * R + 3)
    slots, positions, cu_new, cu_len, lengths_out, n_free_out = both.split((rows, rows, R + 1, R + 1, R, 1))
    table_out, free_out = new_ints((R, W)), new_ints(F)
    at = both.data_ptr()
    p = _Plan(lengths.data_ptr(), new.data_ptr(), table.data_ptr(), free.data_ptr(), n_free.data_ptr(), R, W, F, page_tokens, rows,
              at, at + 4 * rows, at + 8 * rows, at + 4 * (2 * rows + R + 1), at + 4 * (2 * rows + 2 * R + 2), table_out.data_ptr(),
              free_out.data_ptr(), at + 4 * (2 * rows + 3 * R + 2), _raw_stream(dev) if stream is None else stream)
    _call(_lib().hyperattn_cache_plan, "hyperattn_cache_plan", dev, C.byref(p))
    return CachePlan(slots, positions, cu_new, cu_len, lengths_out, table_out, free_out, n_free_out)


def cache_store(cache, k, v, slots, stream=None):
    """Puts k, v [rows, kv_heads, d] (bf16 or fp16, any strides) into the cache's slots [rows] (int32; negative: left out)."""
    c = _cache_of(cache)
    dev = cache.device
    _ints(dev, slots=slots)
    if k.dim() != 3 or k.shape != v.shape or k.shape[1:] != (c.kv_heads, c.d) or slots.shape != k.shape[:1]:
        raise HyperAttnError("k and v must be [rows, kv_heads, d] of the cache, slots [rows]")
    if k.dtype != v.dtype or k.device != dev or v.device != dev:
        raise HyperAttnError("k and v must have one dtype and be on the cache's device")
    k, v = _rows(k), _rows(v)
    ks, vs = k.stride(), v.stride()
    _call(_lib().hyperattn_cache_store, "hyperattn_cache_store", dev, C.byref(c), k.data_ptr(), v.data_ptr(), _code(k.dtype, "k"), k.shape[0],
          ks[0], ks[1], vs[0], vs[1], slots.data_ptr(), _raw_stream(dev) if stream is None else stream)


def cache_read(cache, table, cu, rows, first=None, dtype=torch.bfloat16, stream=None):
    """K and V [rows, kv_heads, d] of cached tokens: rows cu[r] .. cu[r + 1] - 1 are tokens first[r] (default 0), first[r] + 1, ... of
    request r; table [requests, width], cu [requests + 1], first [requests]: int32.  What is not in the cache reads as zeros."""
    c = _cache_of(cache)
    dev = cache.device
    _ints(dev, table=table, cu=cu)
    if first is not None:
        _ints(dev, first=first)
    R = table.shape[0]
    if table.dim() != 2 or cu.shape != (R + 1,) or (first is not None and first.shape != (R,)) or rows < 0:
        raise HyperAttnError("table must be [requests, width], cu [requests + 1], first [requests]")
    k = torch.empty((rows, c.kv_heads, c.d), dtype=dtype, device=dev)
    v = torch.empty_like(k)
    _call(_lib().hyperattn_cache_read, "hyperattn_cache_read", dev, C.byref(c), table.data_ptr(), R, table.shape[1], cu.data_ptr(),
          None if first is None else first.data_ptr(), rows, k.data_ptr(), v.data_ptr(), _code(dtype, "the result"),
          _raw_stream(dev) if stream is None else stream)
    return k, v


def cache_attention(q, cache, table, lengths, scale=0.0, out_dtype=None, stream=None):
    """Attention of one query token a request, q [requests, q_heads, d] (bf16 or fp16, any strides), over its cached tokens
    0 .. lengths[r] - 1.  table [requests, width], lengths [requests]: int32.  Returns (out [requests, q_heads, d], lse
    [requests, q_heads]); a request without tokens gets zeros and -inf."""
    c = _cache_of(cache)
    dev = cache.device
    _ints(dev, table=table, lengths=lengths)
    if q.dim() != 3 or q.shape[2] != c.d or q.device != dev or table.dim() != 2 or table.shape[0] != q.shape[0] or lengths.shape != q.shape[:1]:
        raise HyperAttnError("q must be [requests, q_heads, d] on the cache's device, table [requests, width], lengths [requests]")
    q = _rows(q)
    R, H, d = q.shape
    out = torch.empty((R, H, d), dtype=out_dtype or q.dtype, device=dev)
    lse = torch.empty((R, H), dtype=torch.float32, device=dev)
    qs = q.stride()
    p = _CacheAttention(c, q.data_ptr(), qs[0], qs[1], out.data_ptr(), lse.data_ptr(), table.data_ptr(), lengths.data_ptr(), R, table.shape[1], H,
                        _code(q.dtype, "q"), _code(out.dtype, "the result"), scale, None, 0, _raw_stream(dev) if stream is None else stream)
    L = _lib()
    nbytes = C.c_size_t(0)
    _call(L.hyperattn_cache_attention_workspace_bytes, "hyperattn_cache_attention_workspace_bytes", dev, C.byref(p), C.byref(nbytes))
    if nbytes.value:
        ws = torch.empty(nbytes.value, dtype=torch.uint8, device=dev)
        p.workspace, p.workspace_bytes = ws.data_ptr(), nbytes.value
    _call(L.hyperattn_cache_attention, "hyperattn_cache_attention", dev, C.byref(p))
    return out, lse


def prompt_attention(q, k, v, cu_q, cu_k=None, causal=True, scale=0.0, out_dtype=None, stream=None):
    """Exact attention over packed prompts: q [q_rows, q_heads, d], k, v [k_rows, kv_heads, d] (bf16 or fp16, any strides); request r's
    queries are rows cu_q[r] .. cu_q[r + 1] - 1, its keys rows cu_k[r] .. cu_k[r + 1] - 1 (default: those of the queries).  causal: a
    request's last query sees all its keys, every earlier one a key less.  Returns (out [q_rows, q_heads, d], lse [q_rows,
    q_heads]); a query that sees no key gets zeros and -inf, rows beyond cu_q[-1] are not written."""
    if not q.is_cuda:
        raise HyperAttnError("q, k, v must be CUDA tensors (there is no CPU path)")
    dev = q.device
    cu_k = cu_q if cu_k is None else cu_k
    _ints(dev, cu_q=cu_q, cu_k=cu_k)
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or k.shape[2] != q.shape[2] or cu_q.dim() != 1 or cu_q.numel() < 1 or cu_k.shape != cu_q.shape:
        raise HyperAttnError("q must be [q_rows, q_heads, d], k and v [k_rows, kv_heads, d], cu_q and cu_k [requests + 1]")
    if k.dtype != q.dtype or v.dtype != q.dtype or k.device != dev or v.device != dev:
        raise HyperAttnError("q, k and v must have one dtype and device")
    q, k, v = _rows(q), _rows(k), _rows(v)
    T, H, d = q.shape
    out = torch.empty((T, H, d), dtype=out_dtype or q.dtype, device=dev)
    lse = torch.empty((T, H), dtype=torch.float32, device=dev)
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    p = _Prompt(q.data_ptr(), k.data_ptr(), v.data_ptr(), qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], out.data_ptr(), lse.data_ptr(), cu_q.data_ptr(),
                cu_k.data_ptr(), cu_q.shape[0] - 1, T, k.shape[0], H, k.shape[1], d, 1 if causal else 0, _code(q.dtype, "q"),
                _code(out.dtype, "the result"), scale, _raw_stream(dev) if stream is None else stream)
    _call(_lib().hyperattn_prompt_attention, "hyperattn_prompt_attention", dev, C.byref(p))
    return out, lse
