"""Attention of several new tokens a request over the paged 4-bit cache, and the weight that cached tokens get, against plain 64-bit statements."""
import math

import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (4, 4, 64), (6, 2, 64), (16, 1, 128), (7, 1, 64), (9, 3, 128), (40, 2, 64)]
# lengths after the step and new tokens of the requests: single tokens, tile and page ends, more new tokens than there are, none at all
BATCHES = {
    "one": ([1], [1]),
    "small": ([5, 64, 0, 17, 129, 3], [2, 64, 0, 1, 3, 5]),
    "ends": ([63, 64, 65, 127, 128, 129, 15, 16], [1, 2, 65, 3, 128, 4, 15, 0]),
    "parts": ([300, 200, 1000, 515], [130, 200, 33, 257]),
}


def queries(T, heads, d, dtype, seed=1, scale=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(T, heads, d, generator=gen, device="cuda") * scale).to(dtype)


def both(lens, counts, heads, page, dtype, causal=True, seed=0, q_scale=1.0, out_dtype=None, **kw):
    hq, hkv, d = heads
    cache, table, k, v = CU.filled(lens, hkv, d, page, dtype, seed, **kw)
    q = queries(sum(counts), hq, d, dtype, seed + 1, q_scale)
    got = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts), causal=causal, out_dtype=out_dtype)
    want = CU.attention(q.double(), k, v, lens, counts, causal)
    CU.check_attention(got, want, out_dtype or dtype, max(lens), sum(counts))
    return q, cache, table, k, v, got, want


def check_weights(q, cache, table, k, lens, counts, lse, causal=True, before=None, decay=1.0, there=None):
    cap = table.shape[1] * cache.shape[2] * 16
    got = ha.cache_weights(q, cache, table, CU.ints(lens), lse, CU.offsets(counts), weights=before, decay=decay, causal=causal)
    want, bound = CU.weights(q.double(), k, lens, counts, lse, before, decay, causal, cap=cap, there=there)
    assert got.shape == want.shape and torch.equal(torch.isnan(got), torch.isnan(want))
    fine = ~torch.isnan(want)
    err = torch.where(fine, (got.double() - want).abs(), 0.0)
    assert bool((err <= bound)[fine].all()), float((err / bound)[fine & (bound > 0)].max())
    return got


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("batch", BATCHES)
def test_chunks_and_their_weights(heads, batch):
    lens, counts = BATCHES[batch]
    dtype, page = (torch.bfloat16, 64) if heads[0] % 4 == 0 else (torch.float16, 16)
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, heads, page, dtype)
    before = torch.rand(len(lens), heads[1], table.shape[1] * page, device="cuda")
    check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.75)
    check_weights(q, cache, table, k, lens, counts, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,page", [((8, 2, 64), 32), ((8, 8, 128), 128), ((12, 1, 128), 16), ((4, 2, 64), 1024), ((2, 2, 128), 48)])
def test_full_attention_and_fp32_results(heads, page, dtype):
    lens, counts = [0, 3, 200, 77], [2, 5, 70, 150]
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, heads, page, CU.TYPES[dtype], causal=False, out_dtype=torch.float32)
    assert out.dtype is torch.float32
    check_weights(q, cache, table, k, lens, counts, lse, causal=False)


@pytest.mark.parametrize("heads,lens,counts", [((2, 1, 64), [131072], [3]), ((8, 2, 128), [70001, 31, 9000], [5, 31, 300]), ((4, 1, 128), [20000], [513]), ((1, 1, 64), [33000], [1000])])
def test_long_contexts(heads, lens, counts):
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, heads, 64, torch.float16)
    before = torch.rand(len(lens), heads[1], table.shape[1] * 64, device="cuda")
    check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.5)


def test_one_row_a_request():
    lens, heads = [40, 0, 7, 1000], (8, 2, 128)
    cache, table, k, v = CU.filled(lens, 2, 128, 16)
    q = queries(4, 8, 128, torch.bfloat16)
    got = ha.cache_chunk_attention(q, cache, table, CU.ints(lens))
    want = CU.attention(q.double(), k, v, lens, [1] * 4)
    CU.check_attention(got, want, torch.bfloat16, 1000, 4)
    assert not got[0][1].any() and bool((got[1][1] == -math.inf).all())
    w = ha.cache_weights(q, cache, table, CU.ints(lens), got[1])
    assert torch.equal(w, ha.cache_weights(q, cache, table, CU.ints(lens), got[1], CU.offsets([1] * 4)))
    # all weight of a row goes somewhere: its softmax sums to one, a key head has four rows
    assert torch.allclose(w.sum(-1), torch.tensor([4.0, 0, 4, 4], device="cuda")[:, None].expand(4, 2), atol=1e-4)


def test_rows_beyond_the_last_request_stay():
    lens, counts, T = [30, 50], [3, 4], 12
    cache, table, k, v = CU.filled(lens, 2, 64, 16)
    q = queries(T, 4, 64, torch.bfloat16)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
    want = CU.attention(q[:7].double(), k, v, lens, counts)
    CU.check_attention((out, lse), want, torch.bfloat16, 50, 7)
    w = ha.cache_weights(q, cache, table, CU.ints(lens), lse.nan_to_num(nan=7.0), CU.offsets(counts))
    assert bool(torch.isfinite(w).all())
    # offsets beyond the rows are cut
    cut = ha.cache_chunk_attention(q[:5], cache, table, CU.ints(lens), CU.offsets(counts))
    assert torch.equal(cut[0][:3], out[:3])


def test_no_rows_and_no_requests():
    cache, table, k, v = CU.filled([20], 2, 64, 16)
    q = queries(0, 4, 64, torch.bfloat16)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints([20]), CU.ints([0, 0]))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    before = torch.rand(1, 2, table.shape[1] * 16, device="cuda")
    w = ha.cache_weights(q, cache, table, CU.ints([20]), lse, CU.ints([0, 0]), weights=before, decay=0.5)
    assert torch.equal(w[..., :20], before[..., :20] * 0.5) and not w[..., 20:].any()
    none = ha.cache_chunk_attention(q, cache, table[:0], CU.ints([]), CU.ints([0]))
    assert none[0].shape == (0, 4, 64)
    assert ha.cache_weights(q, cache, table[:0], CU.ints([]), lse, CU.ints([0])).shape == (0, 2, table.shape[1] * 16)


def test_strides_and_addresses():
    lens, counts = [70, 33], [9, 33]
    cache, table, k, v = CU.filled(lens, 2, 64, 16, torch.float16)
    wide = queries(42, 12, 64, torch.float16)
    odd = torch.zeros(42 * 8 * 64 + 3, dtype=torch.float16, device="cuda")[3:].view(42, 8, 64)
    odd.copy_(wide[:, 2:10])
    for q in (wide[:, 2:10], wide.transpose(0, 1).contiguous().transpose(0, 1)[:, 2:10], odd, wide[:, 2:10].flip(0).flip(0), wide[:, ::1][:, 2:10]):
        got = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
        want = CU.attention(q.double(), k, v, lens, counts)
        CU.check_attention(got, want, torch.float16, 70, 42)
        check_weights(q, cache, table, k, lens, counts, got[1])
    lse = torch.stack([got[1], got[1]], -1)[..., 0]                                   # not contiguous
    assert torch.equal(ha.cache_weights(q, cache, table, CU.ints(lens), lse, CU.offsets(counts)), ha.cache_weights(q, cache, table, CU.ints(lens), got[1], CU.offsets(counts)))


def test_missing_pages_hold_nothing():
    lens, counts, page = [100, 200, 40], [7, 130, 40], 16
    cache, table, k, v = CU.filled(lens, 2, 128, page)
    there = torch.ones(sum(lens), dtype=torch.bool, device="cuda")
    for r, c, junk in ((0, 2, -1), (1, 0, -5), (1, 5, 1 << 20), (1, 6, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1)):
        table[r, c] = junk
        a = sum(lens[:r])
        there[a + c * page:a + min((c + 1) * page, lens[r])] = False
    q = queries(sum(counts), 8, 128, torch.bfloat16)
    got = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
    want = CU.attention(q.double(), k, v, lens, counts, there=there)
    CU.check_attention(got, want, torch.bfloat16, 200, sum(counts))
    assert bool((got[1][137:] == -math.inf).all()) and not got[0][137:].any()
    before = torch.rand(3, 2, table.shape[1] * page, device="cuda")
    check_weights(q, cache, table, k, lens, counts, got[1], before=before, decay=0.9, there=there)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("k_scale,v_scale,q_scale", [(1.0, 1e-5, 1.0), (1e-4, 1.0, 1e4), (2e3, 1e4, 1e-3), (1e-5, 3e-6, 1.0), (1.0, 1.0, 30.0), (8e3, 1e-7, 1e-5)])
def test_values_of_any_size(dtype, k_scale, v_scale, q_scale):
    """Scales and minima of the cache are fp16 numbers (steps of 2^-24 below 2^-14), whatever is stored; what they stand for is what counts here."""
    lens, counts = [90, 300], [20, 140]
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, (8, 2, 64), 16, CU.TYPES[dtype], q_scale=q_scale, k_scale=k_scale, v_scale=v_scale)
    check_weights(q, cache, table, k, lens, counts, lse)


@pytest.mark.parametrize("first", [0, 64, 170, 290])
def test_values_whose_size_changes(first):
    """Values 2^-20 to 2^15 in one context, in either order; keys too."""
    def put(k, v):
        n = k.shape[0]
        v[first:] *= 2.0 ** 12
        v[:first // 2] *= 2.0 ** -14
        k[first:first + 40] *= 20
        k[n - 30:] *= 2.0 ** -9
    for heads, dtype in (((8, 2, 64), torch.float16), ((3, 1, 128), torch.bfloat16)):
        q, cache, table, k, v, (out, lse), _ = both([300], [150], heads, 16, dtype, put=put)
        check_weights(q, cache, table, k, [300], [150], lse)


@pytest.mark.parametrize("heads,counts", [((8, 2, 128), [60]), ((4, 4, 64), [3]), ((6, 1, 64), [200])])
def test_groups_that_are_not_numbers(heads, counts):
    """A NaN is a query's own matter: those that see the token have it, others do not."""
    length = 260
    spots = [(length - 5, 0, 3), (length - 20, heads[1] - 1, heads[2] - 1), (length - counts[0] // 2 - 1, 0, 33)]

    def values(k, v):
        for t, h, x in spots:
            v[t, h, x] = math.nan

    both([length], counts, heads, 16, torch.bfloat16, put=values)

    def keys(k, v):
        k[length - 2, 0, 40] = math.inf

    q, cache, table, k, v, (out, lse), want = both([length], counts, heads, 16, torch.float16, put=keys)
    check_weights(q, cache, table, k, [length], counts, torch.where(torch.isnan(lse), 3.0, lse))


def test_queries_that_are_not_numbers():
    lens, counts = [100], [20]
    cache, table, k, v = CU.filled(lens, 2, 64, 16)
    q = queries(20, 8, 64, torch.bfloat16)
    clean = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
    q[5, 3, 7], q[11, 0, 0] = math.nan, math.inf
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
    bad = torch.zeros(20, 8, dtype=torch.bool, device="cuda")
    bad[5, 3] = bad[11, 0] = True
    assert bool(torch.isnan(out[5, 3]).all()) and bool(torch.isnan(lse[5, 3]))
    assert torch.equal(out[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])


def test_a_score_far_above_all_others():
    """References that have to move late, by a lot."""
    def put(k, v):
        k[-1] *= 60
        k[150] *= 30
    for dtype in (torch.float16, torch.bfloat16):
        both([700], [64], (4, 1, 64), 64, dtype, q_scale=3.0, put=put)


def test_twice_the_same_and_beside_others():
    """Runs are equal bit for bit."""
    lens, counts = [1000, 64, 2000, 7], [100, 64, 5, 7]
    q, cache, table, k, v, got, _ = both(lens, counts, (8, 2, 128), 64, torch.bfloat16)
    for _ in range(3):
        again = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
        assert torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    a, b = (ha.cache_weights(q, cache, table, CU.ints(lens), got[1], CU.offsets(counts)) for _ in range(2))
    assert torch.equal(a, b)


def test_weights_in_place():
    lens, counts = [90, 33], [10, 33]
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, (4, 2, 64), 16, torch.bfloat16)
    w = torch.rand(2, 2, table.shape[1] * 16, device="cuda")
    want = ha.cache_weights(q, cache, table, CU.ints(lens), lse, CU.offsets(counts), weights=w, decay=0.25)
    got = ha.cache_weights(q, cache, table, CU.ints(lens), lse, CU.offsets(counts), weights=w, decay=0.25, out=w)
    assert got is w and torch.equal(w, want)


def test_other_streams_and_graphs():
    lens, counts = [500, 40], [100, 3]
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, (8, 2, 64), 16, torch.float16)
    lengths, cu = CU.ints(lens), CU.offsets(counts)
    w = ha.cache_weights(q, cache, table, lengths, lse, cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ha.cache_chunk_attention(q, cache, table, lengths, cu, stream=side.cuda_stream)
    got_w = ha.cache_weights(q, cache, table, lengths, got[1], cu, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], out) and torch.equal(got[1], lse) and torch.equal(got_w, w)
    # two graphs, with other lengths, replayed in turn
    graphs = []
    for ls in (lens, [300, 39]):
        ln = CU.ints(ls)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, l = ha.cache_chunk_attention(q, cache, table, ln, cu)
            ww = ha.cache_weights(q, cache, table, ln, l, cu)
        graphs.append((graph, ln, o, l, ww, ls))
    for _ in range(2):
        for graph, ln, o, l, ww, ls in graphs:
            graph.replay()
            torch.cuda.synchronize()
            eo, el = ha.cache_chunk_attention(q, cache, table, ln, cu)
            assert torch.equal(o, eo) and torch.equal(l, el) and torch.equal(ww, ha.cache_weights(q, cache, table, ln, el, cu))


def test_many_requests():
    gen = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 90, (1000,), generator=gen).tolist()
    counts = [int(x) for x in torch.randint(0, 4, (1000,), generator=gen)]
    q, cache, table, k, v, (out, lse), _ = both(lens, counts, (4, 2, 64), 16, torch.bfloat16)
    check_weights(q, cache, table, k, lens, counts, lse)
