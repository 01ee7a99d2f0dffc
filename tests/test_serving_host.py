"""Refusals of the serving entry points, by the library before anything is launched and by the binding; no GPU needed."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
from paper_2310_05869_b200 import serving as S
import serving_util as SU

AT = 0x10000          # an address that nothing looks at


def cache(**kw):
    return S._Cache(*{**dict(pages=AT, num_pages=10, page_tokens=64, kv_heads=2, d=128), **kw}.values())


BAD_CACHES = [(dict(pages=0), -1), (dict(num_pages=0), -1), (dict(kv_heads=0), -1), (dict(d=96), -2), (dict(page_tokens=24), -2),
              (dict(page_tokens=2048), -2), (dict(num_pages=1 << 26), -2), (dict(pages=AT + 8), -3)]


def plan(**kw):
    names = [n for n, _ in S._Plan._fields_]
    base = {n: AT + 0x1000 * i for i, n in enumerate(names)}
    base.update(requests=4, table_width=8, num_free=10, page_tokens=64, rows=5, stream=None)
    return S._Plan(*[{**base, **kw}[n] for n in names])


@pytest.mark.parametrize("kw,code", [(dict(requests=-1), -1), (dict(table_width=0), -1), (dict(rows=-1), -1), (dict(page_tokens=0), -1), (dict(num_free=-1), -1),
                                     (dict(requests=4097), -2), (dict(table_width=1 << 26), -2), (dict(lengths=None), -1), (dict(slots=None), -1),
                                     (dict(free_pages=None), -1), (dict(n_free_out=None), -1), (dict(table_out=AT + 0x2000), -3), (dict(requests=0), 0)])
def test_plan(kw, code):
    assert S._lib().hyperattn_cache_plan(C.byref(plan(**kw))) == code


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches(kw, code):
    c = cache(**kw)
    assert S._lib().hyperattn_cache_store(C.byref(c), AT, AT, 0, 3, 256, 128, 256, 128, AT, None) == code
    assert S._lib().hyperattn_cache_read(C.byref(c), AT, 2, 3, AT, None, 3, AT, AT, 0, None) == code
    assert S._lib().hyperattn_cache_attention(C.byref(attend(cache=c))) == code


@pytest.mark.parametrize("args,code", [((None, AT, 0, 3, 256, 128, 256, 128, AT), -1), ((AT, AT, 1, 3, 256, 128, 256, 128, AT), -2), ((AT, AT, 7, 3, 256, 128, 256, 128, AT), -1),
                                       ((AT, AT, 0, -3, 256, 128, 256, 128, AT), -1), ((AT, AT, 0, 3, 250, 128, 256, 128, AT), -2), ((AT, AT, 0, 3, 256, 128, 256, -128, AT), -2),
                                       ((AT + 2, AT, 0, 3, 256, 128, 256, 128, AT), -3), ((AT, AT, 2, 3, 256, 128, 256, 128, None), -1), ((None, None, 2, 0, 256, 128, 256, 128, None), 0)])
def test_store(args, code):
    c = cache()
    assert S._lib().hyperattn_cache_store(C.byref(c), *args, None) == code


@pytest.mark.parametrize("args,code", [((AT, 2, 0, AT, None, 3, AT, AT, 0), -1), ((None, 2, 3, AT, None, 3, AT, AT, 0), -1), ((AT, 2, 3, None, None, 3, AT, AT, 0), -1),
                                       ((AT, 2, 3, AT, None, 3, AT, AT + 4, 0), -3), ((AT, 2, 3, AT, None, 3, AT, AT, 5), -1), ((AT, -2, 3, AT, None, 3, AT, AT, 0), -1),
                                       ((AT, 2, 3, AT, None, 0, None, None, 1), 0)])
def test_read(args, code):
    c = cache()
    assert S._lib().hyperattn_cache_read(C.byref(c), *args, None) == code


def attend(**kw):
    names = [n for n, _ in S._CacheAttention._fields_]
    base = dict(cache=cache(), q=AT, q_row_stride=1024, q_head_stride=128, out=AT + 0x1000, lse=AT + 0x2000, table=AT, lengths=AT, requests=3, table_width=9,
                q_heads=8, dtype=0, out_dtype=0, softmax_scale=0.0, workspace=AT, workspace_bytes=1 << 40, stream=None)
    return S._CacheAttention(*[{**base, **kw}[n] for n in names])


@pytest.mark.parametrize("kw,code", [(dict(requests=-1), -1), (dict(table_width=0), -1), (dict(q_heads=0), -1), (dict(q_heads=7), -2), (dict(dtype=1), -2), (dict(dtype=9), -1),
                                     (dict(out_dtype=2), -1), (dict(q_row_stride=1020), -2), (dict(q_head_stride=-8), -2), (dict(q=None), -1), (dict(lse=None), -1),
                                     (dict(lengths=None), -1), (dict(q=AT + 4), -3), (dict(out=AT + 4), -3), (dict(table_width=1 << 26), -2), (dict(requests=0), 0)])
def test_cache_attention(kw, code):
    assert S._lib().hyperattn_cache_attention(C.byref(attend(**kw))) == code


def prompt(**kw):
    names = [n for n, _ in S._Prompt._fields_]
    base = dict(q=AT, k=AT + 0x1000, v=AT + 0x2000, q_row_stride=512, q_head_stride=128, k_row_stride=256, k_head_stride=128, v_row_stride=256, v_head_stride=128, out=AT + 0x3000,
                lse=AT + 0x4000, cu_q=AT, cu_k=AT, requests=2, q_rows=5, k_rows=6, q_heads=4, kv_heads=2, d=128, causal=1, dtype=0, out_dtype=0, softmax_scale=0.0, stream=None)
    return S._Prompt(*[{**base, **kw}[n] for n in names])


@pytest.mark.parametrize("kw,code", [(dict(requests=-1), -1), (dict(q_rows=-1), -1), (dict(q_heads=0), -1), (dict(q_heads=5), -2), (dict(q_heads=258), -2), (dict(d=80), -2),
                                     (dict(dtype=1), -2), (dict(dtype=3), -1), (dict(out_dtype=2), -1), (dict(k_row_stride=4), -2), (dict(v_head_stride=-128), -2), (dict(q=None), -1),
                                     (dict(v=None), -1), (dict(cu_k=None), -1), (dict(lse=None), -1), (dict(k=AT + 2), -3), (dict(out=AT), -3), (dict(q_rows=0), 0), (dict(requests=0), 0)])
def test_prompt(kw, code):
    assert S._lib().hyperattn_prompt_attention(C.byref(prompt(**kw))) == code


def test_the_binding_refuses():
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_plan(i, i, i.view(2, 1), i, i[:1], 64, 3)                              # not on a GPU
    with pytest.raises(ha.HyperAttnError):
        ha.cache_pages(3, 2, 96)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_pages(3, 2, 64, page_tokens=20)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ha.HyperAttnError):
        ha.prompt_attention(x, x, x, i)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_store(torch.zeros(3, 2, 4, 1280, dtype=torch.uint8), x, x, i)
    with pytest.raises(ha.HyperAttnError):
        ha.cache_attention(x, torch.zeros(3, 2, 4, 1281, dtype=torch.uint8), i.view(2, 1), i)


def test_the_plain_statements():
    """The statements that the GPU tests compare with: what is held is within half a step of what was stored, a step a 15th of the group's range."""
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((7, 128)) * 3).astype(np.float16).astype(np.float32)
    got, g = SU.held(x), x.reshape(7, 4, 32)
    step = (g.max(-1) - g.min(-1)) / 15
    assert np.all(np.abs(got - x).reshape(7, 4, 32) <= (0.5 + 16 * 2.0 ** -11) * step[..., None] + 1e-7)
    flat = SU.held(np.full((1, 64), 2.5, np.float32))
    assert np.all(flat == 2.5)
    out, lse, _, _ = SU.attention(np.ones((2, 4)), np.zeros((3, 4)), np.eye(3, 4), [0, 2])
    assert not out[0].any() and lse[0] == -np.inf and np.allclose(out[1], [0.5, 0.5, 0, 0]) and np.isclose(lse[1], np.log(2))
    got = SU.plan([3, 20], [1, -1], [[5, -1], [6, 7]], [8, -1, -1], 1, 16, 3)
    assert got["table"] == [[5, -1], [-1, -1]] and got["slots"] == [83, -1, -1] and got["free"] == [8, 6, 7] and got["n_free"] == [3]


@pytest.mark.parametrize("kw,code", [(dict(page_tokens=1, table_width=1 << 28), -2), (dict(requests=4096, table_width=1 << 19), -2), (dict(requests=1, table_width=1 << 20, num_free=(1 << 31) - (1 << 20)), -2)])
def test_plans_whose_pages_do_not_fit_an_int(kw, code):
    assert S._lib().hyperattn_cache_plan(C.byref(plan(**kw))) == code
