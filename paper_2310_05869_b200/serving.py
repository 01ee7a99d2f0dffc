"""Binding of the serving entry points: exact attention over packed prompts, and a paged cache that holds keys and values in
4 bits, with its scheduling.  Argument marshalling only, like `binding.py`; lengths, tables and slots are int32 CUDA tensors
that only the kernels read, so nothing here waits for the GPU.  `stream`: the handle of a stream to do all of the call on instead of torch's current
one - copies of tensors whose strides do not suit and the memory of results included, as if it were the current one.  The caller orders it with what makes
the arguments and what uses the results; their memory is kept for both streams.

A cache is a uint8 tensor [pages, kv_heads, page_tokens / 16, 20 d] (`cache_pages` makes one; include/hyperattn.h has the order of
its bytes).  A decode step of a server:

    plan = cache_plan(lengths, new, table, free, n_free, page_tokens, rows)       # pages, slots and positions of the step's tokens
    cache_store(cache, k, v, plan.slots)                                          # for every layer: the new keys and values,
    out, lse = cache_attention(q, cache, plan.table, plan.lengths)                # attention over all that is cached
"""
from __future__ import annotations

import ctypes as C
import functools
import struct
from typing import NamedTuple

import torch

from .binding import BF16, FP32, HyperAttnError, _check, _on_stream, lib

FP16 = 2
_CODES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
PLAN_MAX_REQUESTS = 4096


class _Cache(C.Structure):                             # hyperattn_cache
    _fields_ = [("pages", C.c_void_p), ("num_pages", C.c_int), ("page_tokens", C.c_int), ("kv_heads", C.c_int), ("d", C.c_int)]


class _Plan(C.Structure):                              # hyperattn_plan
    _fields_ = ([(n, C.c_void_p) for n in ("lengths", "new_tokens", "table", "free_pages", "n_free")]
                + [(n, C.c_int) for n in ("requests", "table_width", "num_free", "page_tokens", "rows")]
                + [(n, C.c_void_p) for n in ("slots", "positions", "cu_new", "cu_lengths", "lengths_out", "table_out", "free_out",
                                             "n_free_out", "stream")])


class _CacheAttention(C.Structure):                    # hyperattn_cache_attention_params
    _fields_ = [("cache", _Cache), ("q", C.c_void_p), ("q_row_stride", C.c_longlong), ("q_head_stride", C.c_longlong),
                ("out", C.c_void_p), ("lse", C.c_void_p), ("table", C.c_void_p), ("lengths", C.c_void_p),
                ("requests", C.c_int), ("table_width", C.c_int), ("q_heads", C.c_int), ("dtype", C.c_int), ("out_dtype", C.c_int),
                ("softmax_scale", C.c_float), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("stream", C.c_void_p)]


class _Prompt(C.Structure):                            # hyperattn_prompt_params
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v")]
                + [(n, C.c_longlong) for n in ("q_row_stride", "q_head_stride", "k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")]
                + [(n, C.c_void_p) for n in ("out", "lse", "cu_q", "cu_k")]
                + [(n, C.c_int) for n in ("requests", "q_rows", "k_rows", "q_heads", "kv_heads", "d", "causal", "dtype", "out_dtype")]
                + [("softmax_scale", C.c_float), ("stream", C.c_void_p)])


def _packer(kind):
    """A struct's members as bytes: what a call passes (filling a ctypes object member by member takes several times as long)."""
    def format_of(kind):
        letters = {C.c_void_p: "P", C.c_int: "i", C.c_longlong: "q", C.c_float: "f", C.c_size_t: "N"}
        return "".join(letters[t] if t in letters else format_of(t) + "0P" for _, t in kind._fields_)
    packer = struct.Struct("@" + format_of(kind))
    assert packer.size == C.sizeof(kind)
    return packer.pack


_cache_bytes, _plan_bytes, _attention_bytes, _prompt_bytes = (_packer(k) for k in (_Cache, _Plan, _CacheAttention, _Prompt))


@functools.cache
def _lib():
    L = lib()
    i, p, ll = C.c_int, C.c_void_p, C.c_longlong
    for name, args in (("hyperattn_cache_plan", [p]), ("hyperattn_cache_store", [p, p, p, i, i, ll, ll, ll, ll, p, p]),
                       ("hyperattn_cache_read", [p, p, i, i, p, p, i, p, p, i, p]), ("hyperattn_cache_attention", [p]),
                       ("hyperattn_cache_attention_workspace_bytes", [p, C.POINTER(C.c_size_t)]), ("hyperattn_prompt_attention", [p])):
        getattr(L, name).restype = i
        getattr(L, name).argtypes = args
    return L


def _call(name, index, *args):
    """Calls an entry point with device `index` current."""
    fn = getattr(_lib(), name)
    if torch._C._cuda_getDevice() == index:
        rc = fn(*args)
    else:
        with torch.cuda.device(index):
            rc = fn(*args)
    if rc:
        _check(rc, name)


_stream = torch._C._cuda_getCurrentRawStream


def _new(shape, dtype, device):
    """torch.empty of one to three axes (which takes longer to find out that the strides are these)."""
    if len(shape) == 3:
        return torch.empty_strided(shape, (shape[1] * shape[2], shape[2], 1), dtype=dtype, device=device)
    return torch.empty_strided(shape, (shape[1], 1) if len(shape) == 2 else (1,), dtype=dtype, device=device)


def _ints(index, *tensors):
    """The int32 tensors of a call: on its device, contiguous."""
    for t in tensors:
        if t.dtype is not torch.int32 or t.get_device() != index or not t.is_contiguous():
            raise HyperAttnError("lengths, offsets, tables and slots must be contiguous int32 tensors on the device of the call")


def _rows(x):
    """x [rows, heads, d] and its row and head strides as the kernels take them: d contiguous, the others and the address in steps of 16 bytes."""
    row, head, one = x.stride()
    if one != 1 or row % 8 or head % 8 or row <= 0 or head <= 0 or x.data_ptr() % 16:
        x = x.clone(memory_format=torch.contiguous_format)
        row, head, one = x.stride()
    return x, row, head


def _code(t, what):
    code = _CODES.get(t)
    if code is None:
        raise HyperAttnError(f"unsupported dtype {t} of {what}")
    return code


def _cache_of(cache):
    """The members of hyperattn_cache."""
    if cache.dtype is torch.uint8 and cache.is_cuda and cache.dim() == 4 and cache.is_contiguous():
        pages, heads, blocks, size = cache.shape
        if size == 1280 or size == 2560:
            return cache.data_ptr(), pages, blocks * 16, heads, size // 20
    raise HyperAttnError("a cache is a contiguous CUDA uint8 tensor [pages, kv_heads, page_tokens / 16, 20 d], d 64 or 128")


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
    if stream is not None:
        return _on_stream(stream, cache_plan, lengths, new, table, free, n_free, page_tokens, rows)
    if not lengths.is_cuda:
        raise HyperAttnError("lengths must be a CUDA tensor (there is no CPU path)")
    index = lengths.get_device()
    _ints(index, lengths, new, table, free, n_free)
    if lengths.dim() != 1 or table.dim() != 2 or free.dim() != 1 or n_free.numel() != 1 or new.shape != lengths.shape or table.shape[0] != lengths.shape[0]:
        raise HyperAttnError("lengths and new are [requests], table [requests, width], free [pages], n_free [1]")
    if rows < 0 or page_tokens <= 0:
        raise HyperAttnError("rows must not be negative, page_tokens positive")
    R, W = table.shape
    F = free.shape[0]
    if R == 0:
        none = lengths.new_full((2, rows), -1)
        zero = lengths.new_zeros((2, 1))
        left = n_free.clamp(0, F).view(1)
        stack = torch.where(torch.arange(F, dtype=torch.int32, device=free.device) < left, free, -1)
        return CachePlan(none[0], none[1], zero[0], zero[1], lengths.clone(), table.clone(), stack, left)
    # one allocation for all but the table, the stack first (its address stays in steps of 16 bytes)
    flat = _new((F + 2 * rows + 3 * R + 3,), torch.int32, lengths.device)
    table_out = torch.empty_like(table)
    stack = flat.data_ptr()
    at = stack + 4 * F
    _call("hyperattn_cache_plan", index, _plan_bytes(
        lengths.data_ptr(), new.data_ptr(), table.data_ptr(), free.data_ptr(), n_free.data_ptr(), R, W, F, page_tokens, rows,
        at, at + 4 * rows, at + 8 * rows, at + 4 * (2 * rows + R + 1), at + 4 * (2 * rows + 2 * R + 2), table_out.data_ptr(),
        stack, at + 4 * (2 * rows + 3 * R + 2), _stream(index)))
    free_out, slots, positions, cu_new, cu_len, lengths_out, n_free_out = torch.unsafe_split_with_sizes(flat, (F, rows, rows, R + 1, R + 1, R, 1))
    return CachePlan(slots, positions, cu_new, cu_len, lengths_out, table_out, free_out, n_free_out)


def cache_store(cache, k, v, slots, stream=None):
    """Puts k, v [rows, kv_heads, d] (bf16 or fp16, any strides) into the cache's slots [rows] (int32; negative: left out)."""
    if stream is not None:
        return _on_stream(stream, cache_store, cache, k, v, slots)
    c = _cache_of(cache)
    index = cache.get_device()
    _ints(index, slots)
    if k.dim() != 3 or k.shape != v.shape or k.shape[1:] != c[3:] or slots.shape != k.shape[:1]:
        raise HyperAttnError("k and v must be [rows, kv_heads, d] of the cache, slots [rows]")
    if k.dtype is not v.dtype or k.get_device() != index or v.get_device() != index:
        raise HyperAttnError("k and v must have one dtype and be on the cache's device")
    k, k_row, k_head = _rows(k)
    v, v_row, v_head = _rows(v)
    _call("hyperattn_cache_store", index, _cache_bytes(*c), k.data_ptr(), v.data_ptr(), _code(k.dtype, "k"), k.shape[0], k_row, k_head, v_row, v_head,
          slots.data_ptr(), _stream(index))


def cache_read(cache, table, cu, rows, first=None, dtype=torch.bfloat16, stream=None):
    """K and V [rows, kv_heads, d] of cached tokens: rows cu[r] .. cu[r + 1] - 1 are tokens first[r] (default 0), first[r] + 1, ... of
    request r; table [requests, width], cu [requests + 1], first [requests]: int32.  What is not in the cache reads as zeros."""
    if stream is not None:
        return _on_stream(stream, cache_read, cache, table, cu, rows, first, dtype)
    c = _cache_of(cache)
    index = cache.get_device()
    _ints(index, table, cu)
    if table.dim() != 2 or cu.dim() != 1 or cu.shape[0] != table.shape[0] + 1 or rows < 0:
        raise HyperAttnError("table must be [requests, width], cu [requests + 1], first [requests]")
    R, W = table.shape
    if first is not None:
        _ints(index, first)
        if first.dim() != 1 or first.shape[0] != R:
            raise HyperAttnError("table must be [requests, width], cu [requests + 1], first [requests]")
    k = _new((rows, c[3], c[4]), dtype, cache.device)
    v = torch.empty_like(k)
    _call("hyperattn_cache_read", index, _cache_bytes(*c), table.data_ptr(), R, W, cu.data_ptr(), None if first is None else first.data_ptr(), rows,
          k.data_ptr(), v.data_ptr(), _code(dtype, "the result"), _stream(index))
    return k, v


@functools.lru_cache(4096)
def _attention_workspace(*shape):
    """Workspace of hyperattn_cache_attention: (pages, page_tokens, kv_heads, d, requests, width, q_heads, dtype, out_dtype)."""
    size = C.c_size_t(0)
    cache, (R, W, H, dtype, out_dtype) = shape[:4], shape[4:]
    d = cache[3]
    _check(_lib().hyperattn_cache_attention_workspace_bytes(_attention_bytes(
        16, *cache, 0, d, d, 0, 0, 0, 0, R, W, H, dtype, out_dtype, 0.0, 0, 0, 0), C.byref(size)), "hyperattn_cache_attention_workspace_bytes")
    return size.value


def cache_attention(q, cache, table, lengths, scale=0.0, out_dtype=None, stream=None):
    """Attention of one query token a request, q [requests, q_heads, d] (bf16 or fp16, any strides), over its cached tokens
    0 .. lengths[r] - 1.  table [requests, width], lengths [requests]: int32.  Returns (out [requests, q_heads, d], lse
    [requests, q_heads]); a request without tokens gets zeros and -inf."""
    if stream is not None:
        return _on_stream(stream, cache_attention, q, cache, table, lengths, scale, out_dtype)
    c = _cache_of(cache)
    index = cache.get_device()
    _ints(index, table, lengths)
    if q.dim() != 3 or table.dim() != 2 or lengths.dim() != 1 or q.get_device() != index:
        raise HyperAttnError("q must be [requests, q_heads, d] on the cache's device, table [requests, width], lengths [requests]")
    R, H, d = q.shape
    W = table.shape[1]
    if d != c[4] or table.shape[0] != R or lengths.shape[0] != R:
        raise HyperAttnError("q must be [requests, q_heads, d] on the cache's device, table [requests, width], lengths [requests]")
    q, row, head = _rows(q)
    out_dtype = out_dtype or q.dtype
    dtype, out_code = _code(q.dtype, "q"), _code(out_dtype, "the result")
    device = q.device
    out = _new((R, H, d), out_dtype, device)
    lse = _new((R, H), torch.float32, device)
    size = _attention_workspace(*c[1:], R, W, H, dtype, out_code)
    work = _new((size,), torch.uint8, device)
    _call("hyperattn_cache_attention", index, _attention_bytes(
        *c, q.data_ptr(), row, head, out.data_ptr(), lse.data_ptr(), table.data_ptr(), lengths.data_ptr(), R, W, H, dtype, out_code, scale,
        work.data_ptr(), size, _stream(index)))
    return out, lse


def prompt_attention(q, k, v, cu_q, cu_k=None, causal=True, scale=0.0, out_dtype=None, stream=None):
    """Exact attention over packed prompts: q [q_rows, q_heads, d], k, v [k_rows, kv_heads, d] (bf16 or fp16, any strides); request r's
    queries are rows cu_q[r] .. cu_q[r + 1] - 1, its keys rows cu_k[r] .. cu_k[r + 1] - 1 (default: those of the queries).  causal: a
    request's last query sees all its keys, every earlier one a key less.  Returns (out [q_rows, q_heads, d], lse [q_rows,
    q_heads]); a query that sees no key gets zeros and -inf, rows beyond cu_q[-1] are not written."""
    if stream is not None:
        return _on_stream(stream, prompt_attention, q, k, v, cu_q, cu_k, causal, scale, out_dtype)
    if not q.is_cuda:
        raise HyperAttnError("q, k, v must be CUDA tensors (there is no CPU path)")
    index = q.get_device()
    cu_k = cu_q if cu_k is None else cu_k
    _ints(index, cu_q, cu_k)
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or cu_q.dim() != 1 or cu_q.shape[0] < 1 or cu_k.shape != cu_q.shape:
        raise HyperAttnError("q must be [q_rows, q_heads, d], k and v [k_rows, kv_heads, d], cu_q and cu_k [requests + 1]")
    if k.dtype is not q.dtype or v.dtype is not q.dtype or k.get_device() != index or v.get_device() != index:
        raise HyperAttnError("q, k and v must have one dtype and device")
    T, H, d = q.shape
    k_rows, kv_heads, k_d = k.shape
    if k_d != d:
        raise HyperAttnError("q, k and v must have one head dimension")
    q, q_row, q_head = _rows(q)
    k, k_row, k_head = _rows(k)
    v, v_row, v_head = _rows(v)
    out_dtype = out_dtype or q.dtype
    dtype, out_code = _code(q.dtype, "q"), _code(out_dtype, "the result")
    device = q.device
    out = _new((T, H, d), out_dtype, device)
    lse = _new((T, H), torch.float32, device)
    _call("hyperattn_prompt_attention", index, _prompt_bytes(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), q_row, q_head, k_row, k_head, v_row, v_head, out.data_ptr(), lse.data_ptr(), cu_q.data_ptr(),
        cu_k.data_ptr(), cu_q.shape[0] - 1, T, k_rows, H, kv_heads, d, 1 if causal else 0, dtype, out_code, scale, _stream(index)))
    return out, lse
