"""Sizes whose indexes would pass 31 bits are refused; no GPU needed."""
import ctypes as C

import pytest

from paper_2310_05869_b200 import serving as S
import test_chunk_host as TH

NEAR = (1 << 31) - (1 << 16)          # places of a table row


@pytest.mark.parametrize("width,page", [(NEAR // 16, 16), (NEAR // 64, 64), ((1 << 31) // 64 - 1, 64), ((1 << 31) // 1024 - 1, 1024)])
def test_tables_of_nearly_2_31_places(width, page):
    size = C.c_size_t(0)
    kw = dict(cache=TH.cache(page_tokens=page, kv_heads=1), table_width=width)
    for name, p in (("chunk_attention", TH.chunk(**kw)), ("weights", TH.weights(**kw))):
        assert getattr(S._lib(), f"hyperattn_cache_{name}_workspace_bytes")(C.byref(p), C.byref(size)) == -2
        assert getattr(S._lib(), f"hyperattn_cache_{name}")(C.byref(p)) == -2
    assert S._lib().hyperattn_cache_evict(C.byref(TH.evict(requests=1, **kw))) == -2


@pytest.mark.parametrize("kw", [dict(num_free=(1 << 31) - 33), dict(num_free=(1 << 31) - (1 << 20)), dict(requests=4096, table_width=(1 << 19) - 8)])
def test_plans_of_nearly_2_31_entries(kw):
    assert S._lib().hyperattn_cache_evict_plan(C.byref(TH.plan(**kw))) == -2


def test_workspaces_of_the_largest_tables():
    """Tables just below the limit are taken, and their workspaces do not follow the tokens."""
    size = C.c_size_t(0)
    for rows in (7, 4000):
        for name, make in (("chunk_attention", TH.chunk), ("weights", TH.weights)):
            p = make(cache=TH.cache(kv_heads=1), table_width=NEAR // 64 - 1, rows=rows)
            assert getattr(S._lib(), f"hyperattn_cache_{name}_workspace_bytes")(C.byref(p), C.byref(size)) == 0
            assert size.value < 1 << 30
