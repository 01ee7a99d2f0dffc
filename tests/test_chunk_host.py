"""Refusals of the entry points that add to a cache and keep it within bounds, by the library before anything is launched and by the binding; no GPU needed."""
import ctypes as C

import pytest
import torch

import paper_2310_05869_b200 as ha
from paper_2310_05869_b200 import serving as S

AT = 0x10000          # an address that nothing looks at


def cache(**kw):
    return S._Cache(*{**dict(pages=AT, num_pages=10, page_tokens=64, kv_heads=2, d=128), **kw}.values())


BAD_CACHES = [(dict(pages=0), -1), (dict(num_pages=0), -1), (dict(kv_heads=0), -1), (dict(d=96), -2), (dict(page_tokens=24), -2),
              (dict(page_tokens=2048), -2), (dict(num_pages=1 << 26), -2), (dict(pages=AT + 8), -3)]


def made(kind, base, kw):
    names = [n for n, _ in kind._fields_]
    return kind(*[{**base, **kw}[n] for n in names])


def chunk(**kw):
    return made(S._Chunk, dict(cache=cache(), q=AT, q_row_stride=1024, q_head_stride=128, out=AT + 0x1000, lse=AT + 0x2000, table=AT, lengths=AT, cu_q=AT, requests=3, rows=7,
                               table_width=9, q_heads=8, causal=1, dtype=0, out_dtype=0, softmax_scale=0.0, workspace=AT, workspace_bytes=1 << 40, stream=None), kw)


COMMON = [(dict(requests=-1), -1), (dict(rows=-1), -1), (dict(table_width=0), -1), (dict(q_heads=0), -1), (dict(q_heads=7), -2), (dict(dtype=1), -2), (dict(dtype=9), -1),
          (dict(q_row_stride=1020), -2), (dict(q_head_stride=-8), -2), (dict(lengths=None), -1), (dict(table=None), -1), (dict(q=AT + 4), -3), (dict(table_width=1 << 26), -2),
          (dict(requests=4097), -2), (dict(rows=1 << 29), -2), (dict(cu_q=None), -1), (dict(requests=0, rows=0), 0)]


@pytest.mark.parametrize("kw,code", COMMON + [(dict(out_dtype=2), -1), (dict(q=None), -1), (dict(lse=None), -1), (dict(out=None), -1), (dict(out=AT + 4), -3), (dict(rows=0), 0)])
def test_chunk(kw, code):
    assert S._lib().hyperattn_cache_chunk_attention(C.byref(chunk(**kw))) == code


def weights(**kw):
    return made(S._Weights, dict(cache=cache(), q=AT, q_row_stride=1024, q_head_stride=128, lse=AT, weights=AT, weights_out=AT, table=AT, lengths=AT, cu_q=AT, requests=3, rows=7,
                                 table_width=9, q_heads=8, causal=1, dtype=0, softmax_scale=0.0, decay=1.0, workspace=AT, workspace_bytes=1 << 40, stream=None), kw)


@pytest.mark.parametrize("kw,code", COMMON + [(dict(q=None), -1), (dict(lse=None), -1), (dict(weights_out=None), -1), (dict(weights=AT + 4), -3), (dict(weights_out=AT + 8), -3)])
def test_weights(kw, code):
    assert S._lib().hyperattn_cache_weights(C.byref(weights(**kw))) == code


def plan(**kw):
    names = [n for n, _ in S._EvictPlan._fields_]
    base = {n: AT + 0x1000 * i for i, n in enumerate(names)}
    base.update(requests=4, table_width=8, num_free=10, page_tokens=64, stream=None)
    return made(S._EvictPlan, base, kw)


@pytest.mark.parametrize("kw,code", [(dict(requests=-1), -1), (dict(table_width=0), -1), (dict(page_tokens=0), -1), (dict(num_free=-1), -1), (dict(requests=4097), -2),
                                     (dict(table_width=1 << 26), -2), (dict(page_tokens=1, table_width=1 << 28), -2), (dict(requests=4096, table_width=1 << 19), -2), (dict(keep=None), -1),
                                     (dict(lengths=None), -1), (dict(free_pages=None), -1), (dict(n_free_out=None), -1), (dict(table_out=AT + 0x2000), -3),
                                     (dict(lengths_out=AT + 0x1000), -3), (dict(requests=0), 0)])
def test_evict_plan(kw, code):
    assert S._lib().hyperattn_cache_evict_plan(C.byref(plan(**kw))) == code


def evict(**kw):
    return made(S._Evict, dict(cache=cache(), weights=AT, weights_out=AT + 0x1000, kept=AT + 0x2000, table=AT, lengths=AT, to_table=AT, to_lengths=AT, requests=3, table_width=9, recent=4,
                               first=0, stream=None), kw)


@pytest.mark.parametrize("kw,code", [(dict(requests=-1), -1), (dict(table_width=0), -1), (dict(recent=-1), -1), (dict(first=-1), -1), (dict(requests=4097), -2), (dict(table_width=1 << 26), -2),
                                     (dict(weights=None), -1), (dict(kept=None), -1), (dict(to_table=None), -1), (dict(to_lengths=None), -1), (dict(weights_out=AT), -3), (dict(kept=AT + 4), -3),
                                     (dict(requests=0), 0)])
def test_evict(kw, code):
    assert S._lib().hyperattn_cache_evict(C.byref(evict(**kw))) == code


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches(kw, code):
    for fn, p in (("chunk_attention", chunk), ("weights", weights), ("evict", evict)):
        assert getattr(S._lib(), "hyperattn_cache_" + fn)(C.byref(p(cache=cache(**kw)))) == code
    size = C.c_size_t(0)
    assert S._lib().hyperattn_cache_chunk_attention_workspace_bytes(C.byref(chunk(cache=cache(**kw))), C.byref(size)) == code
    assert S._lib().hyperattn_cache_weights_workspace_bytes(C.byref(weights(cache=cache(**kw))), C.byref(size)) == code


def test_workspaces():
    """They follow from the arguments alone, and what is too small is refused."""
    for fn, p in (("chunk_attention", chunk), ("weights", weights)):
        size = C.c_size_t(0)
        assert getattr(S._lib(), f"hyperattn_cache_{fn}_workspace_bytes")(C.byref(p()), C.byref(size)) == 0
        assert getattr(S._lib(), f"hyperattn_cache_{fn}_workspace_bytes")(C.byref(p()), None) == -1
        if size.value:
            assert getattr(S._lib(), f"hyperattn_cache_{fn}")(C.byref(p(workspace_bytes=size.value - 1))) == -4
            assert getattr(S._lib(), f"hyperattn_cache_{fn}")(C.byref(p(workspace=None))) == -1
            assert getattr(S._lib(), f"hyperattn_cache_{fn}")(C.byref(p(workspace=AT + 8))) == -3


def test_the_binding_refuses():
    i = torch.zeros(2, dtype=torch.int32)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    cpu = torch.zeros(3, 2, 4, 1280, dtype=torch.uint8)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_chunk_attention(x, cpu, i.view(2, 1), i)                              # not on a GPU
    with pytest.raises(ha.HyperAttnError):
        ha.cache_weights(x, cpu, i.view(2, 1), i, torch.zeros(2, 2))
    with pytest.raises(ha.HyperAttnError):
        ha.cache_evict_plan(i, i, i.view(2, 1), i, i[:1], 64)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_evict(cpu, torch.zeros(2, 2, 64), i.view(2, 1), i, i.view(2, 1), i)
