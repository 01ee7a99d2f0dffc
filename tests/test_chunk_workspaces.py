"""Workspaces of chunks and weights, on the host: what calls of either kind of kernels and of both need, that what is too small is refused, and what many places of few requests cost."""
import ctypes as C

import pytest

from paper_2310_05869_b200 import serving as S
import test_chunk_host as H

MANY = dict(requests=1, rows=400)                                  # more rows than the few rows' kernels are for
BOTH = dict(requests=64, rows=600, table_width=100)                # 600 tokens of 64 requests, four rows each: all of one, perhaps
FEW = dict(requests=64, rows=64)


def size_of(fn, p):
    size = C.c_size_t(0)
    assert getattr(S._lib(), f"hyperattn_cache_{fn}_workspace_bytes")(C.byref(p), C.byref(size)) == 0
    return size.value


@pytest.mark.parametrize("kw", [MANY, BOTH])
@pytest.mark.parametrize("d", [64, 128])
def test_too_small_and_misplaced_ones(kw, d):
    for fn, p in (("chunk_attention", H.chunk), ("weights", H.weights)):
        kw = dict(kw, cache=H.cache(d=d))
        size = size_of(fn, p(**kw))
        assert size > 0
        for entry in (lambda x: getattr(S._lib(), f"hyperattn_cache_{fn}")(x), lambda x: getattr(S._lib(), f"hyperattn_cache_{fn}_ex")(x, 1)):
            assert entry(C.byref(p(**kw, workspace_bytes=size - 1))) == -4
            assert entry(C.byref(p(**kw, workspace=None))) == -1
            assert entry(C.byref(p(**kw, workspace=H.AT + 8))) == -3


def test_both_kinds_have_room_side_by_side():
    few, both = (size_of("chunk_attention", H.chunk(**kw)) for kw in (FEW, BOTH))
    many = size_of("chunk_attention", H.chunk(**dict(BOTH, requests=1)))
    assert both > many and few > 0
    assert size_of("weights", H.weights(**FEW)) == 0               # (images are the other kernels')


@pytest.mark.parametrize("requests,rows", [(512, 512), (1024, 1024), (4096, 4096), (4096, 70), (64, 2000)])
@pytest.mark.parametrize("heads,kv_heads,d", [(32, 8, 128), (32, 32, 64)])
def test_places_without_many_rows_cost_little(requests, rows, heads, kv_heads, d):
    """An image of queries is some 24 KB a key head.  Requests of up to 16 rows have none, so there are no more of them than a request for every 17 rows, and one for every 96 or 128 rows."""
    size = size_of("weights", H.weights(requests=requests, rows=rows, q_heads=heads, cache=H.cache(kv_heads=kv_heads, d=d)))
    group = rows * heads // kv_heads
    assert size <= (group // 96 + group // 17 + 2) * kv_heads * 29 * 1024


def test_the_most_new_tokens():
    for fn, p in (("chunk_attention", H.chunk), ("weights", H.weights)):
        entry = getattr(S._lib(), f"hyperattn_cache_{fn}_ex")
        assert entry(C.byref(p()), -1) == -1
        assert entry(None, 1) == -1
        assert entry(C.byref(p(requests=0, rows=0)), 5) == 0
    with pytest.raises(S.HyperAttnError):
        S._most(-1)
    assert S._most(None) == 0 and S._most(0) == 1 and S._most(7) == 7 and S._most(1 << 40) == 0x7fffffff
