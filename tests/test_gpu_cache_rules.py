"""Chunks, weights and eviction where one way of computing them ends and another begins, and what only some sizes reach; offsets that do not ascend."""
import math

import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU
import test_gpu_cache_chunk as TC
import test_gpu_cache_evict as TE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("width", [20, 80])
@pytest.mark.parametrize("rows", [4, 5, 8, 9, 16, 17, 32, 33, 64, 65])
def test_around_the_numbers_of_rows_that_decide(rows, width, d):
    """Rows a request on average, tables of more and of fewer than 1024 tokens."""
    lens, counts = [300, 150], [rows, rows]
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, (2, 2, d), 16, torch.float16 if rows % 2 else torch.bfloat16, width=width)
    before = torch.rand(2, 2, width * 16, device="cuda")
    TC.check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.5)


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (3, 1, 64), (16, 1, 128)])
def test_one_request_of_many_rows_beside_many_of_one(heads):
    lens, counts = [300] + [1 + 7 * i for i in range(79)], [70 // (heads[0] // heads[1])] + [1] * 79
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, heads, 16, torch.bfloat16)
    before = torch.rand(80, heads[1], table.shape[1] * 16, device="cuda")
    TC.check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.75)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_very_different_size(d):
    """Rows whose largest entries are up to 2^40 apart: one power of two for all of them would lose the small ones."""
    lens, counts, H = [500], [150], 2
    cache, table, k, v = CU.filled(lens, H, d, 16)
    q = TC.queries(150, 4, d, torch.bfloat16).float()
    q *= torch.exp2(-(torch.arange(600, device="cuda") * 7 % 41).float()).view(150, 4, 1)
    q[17, 2], q[18] = 0, 0
    q = q.to(torch.bfloat16)
    for scale in (0.0, 2.0 ** 30):
        # (queries that are as much smaller as the scale is larger)
        q_now = q if scale == 0.0 else (q.float() * 2.0 ** -30).to(torch.bfloat16)
        out, lse = ha.cache_chunk_attention(q_now, cache, table, CU.ints(lens), CU.offsets(counts), scale=scale)
        want = CU.attention(q_now.double(), k, v, lens, counts, scale=scale or None)
        CU.check_attention((out, lse), want, torch.bfloat16, 500, 150)
        got = ha.cache_weights(q_now, cache, table, CU.ints(lens), lse, CU.offsets(counts), scale=scale)
        exact, bound = CU.weights(q_now.double(), k, lens, counts, lse, scale=scale or None, cap=table.shape[1] * 16)
        assert bool(((got.double() - exact).abs() <= bound).all())


@pytest.mark.parametrize("rows", [100, 128, 356])
@pytest.mark.parametrize("length", [40, 64, 65, 128, 129, 200, 1500])
def test_segments_of_up_to_128_rows(length, rows):
    """Few tiles, odd numbers of them, more rows than tokens; values whose size changes and NaN in tiles of either parity."""
    def sizes(k, v):
        v[: length // 2] *= 2.0 ** -12
        k[length // 3:] *= 8.0

    def nan(k, v):
        v[length - 1, 0, 5] = math.nan
        v[max(length - 70, 0), 0, 40] = math.nan

    for put in (sizes, nan):
        TC.both([length], [rows], (1, 1, 64), 16, torch.float16, width=128, put=put)
        TC.both([length, 70], [rows // 3, 128], (3, 1, 128), 48, torch.bfloat16, width=40, put=put, causal=put is sizes)


@pytest.mark.parametrize("lens,keep", [([400000, 100], [399000, 7]), ([409600], [12345])])
def test_cuts_whose_weights_do_not_fit_a_cluster(lens, keep):
    TE.check(lens, keep, 1, 64, 1024, recent=50, first=4)
    TE.check(lens, keep, 1, 64, 1024, recent=0, first=0, kind="odd")


@pytest.mark.parametrize("rows", [2, 40])
def test_few_tokens_in_wide_tables(rows):
    lens, counts = [5, 0, 4097, 63], [rows] * 4
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, (2, 1, 64), 48, torch.bfloat16, width=700)
    got = TC.check_weights(q, cache, table, k, lens, counts, lse)
    assert not got[1].any() and not got[0, :, 5:].any()


def test_runs_of_operators_in_two_graphs_and_streams_at_once():
    """A step of each of two caches, captured, replayed at the same time on two streams, many times."""
    def step(seed, lens, counts, heads):
        cache, table, k, v = CU.filled(lens, heads[1], heads[2], 16, torch.float16, seed, spare=100)
        q = TC.queries(sum(counts), *heads[::2], torch.float16, seed)
        lengths, cu, keep = CU.ints(lens), CU.offsets(counts), CU.ints([n // 2 for n in lens])
        used = set(table.flatten().tolist())
        free = CU.ints([p for p in range(cache.shape[0]) if p not in used])
        n_free = CU.ints([free.shape[0]])

        def run():
            out, lse = ha.cache_chunk_attention(q, cache, table, lengths, cu)
            w = ha.cache_weights(q, cache, table, lengths, lse, cu)
            plan = ha.cache_evict_plan(lengths, keep, table, free, n_free, 16)
            return (out, lse, w, *plan, *ha.cache_evict(cache, w, table, lengths, plan.table, plan.lengths, 8, 2))
        return run

    runs = [step(1, [500, 40, 300], [100, 3, 1], (8, 2, 64)), step(2, [200] * 9, [2] * 9, (4, 4, 128))]
    want = [[x.clone() for x in run()] for run in runs]
    graphs = []
    for run in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = run()
        graphs.append((graph, got, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, _, stream in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for (_, got, _), exact in zip(graphs, want):
        for x, y in zip(got, exact):
            assert torch.equal(x, y)


@pytest.mark.parametrize("cu,heads", [([0, 40, 0, 40, 5, 40], (4, 2, 64)), ([40, 0, 40, 0, 40, 0], (4, 2, 64)), ([-7, 300, 100, 1000, 0, 2], (16, 2, 128)),
                                      ([0, 300, 0, 300, 0, 300], (8, 1, 64))])
def test_offsets_that_do_not_ascend(cu, heads):
    """Results of requests whose rows are other requests' too are not defined; nothing outside is touched, and the next call is as ever."""
    lens = [100, 50, 0, 70, 300]
    cache, table, k, v = CU.filled(lens, heads[1], heads[2], 16)
    q = TC.queries(300, heads[0], heads[2], torch.bfloat16)
    before = cache.clone()
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.ints(cu))
    ha.cache_weights(q, cache, table, CU.ints(lens), torch.zeros_like(lse), CU.ints(cu))
    torch.cuda.synchronize()
    assert torch.equal(cache, before)
    counts = [60] * 5
    got = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts))
    CU.check_attention(got, CU.attention(q.double(), k, v, lens, counts), torch.bfloat16, 300, 300)


def test_offsets_that_ask_for_more_than_numbers_hold():
    """4096 requests, every other one with all of 131072 rows over 131072 tokens: 2^35 units of work.  None of it is done."""
    cache = ha.cache_pages(4, 1, 64, 1024)
    table = torch.full((4096, 128), -1, dtype=torch.int32, device="cuda")
    q = TC.queries(131072, 1, 64, torch.bfloat16)
    cu = CU.ints([0, 131072] * 2048 + [0])
    out, lse = ha.cache_chunk_attention(q, cache, table, torch.full((4096,), 131072, dtype=torch.int32, device="cuda"), cu)
    torch.cuda.synchronize()
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", [(2, 2, 64), (4, 1, 128), (8, 2, 64)])
def test_a_part_of_a_prompt_beside_single_tokens(heads, causal):
    """Few rows a request on average, and some of many: both kinds of kernels have their requests."""
    G = heads[0] // heads[1]
    lens, counts = [1 + 11 * i for i in range(60)], [1] * 60
    for r, n, length in ((0, 300, 500), (23, 0, 40), (24, 33 // G + 1, 1500), (25, 5, 0), (40, 32 // G, 700), (41, 16 // G, 700), (42, 17 // G + 1, 100), (59, 400 // G, 399 // G)):
        lens[r], counts[r] = length, n
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, heads, 16, torch.bfloat16, causal=causal, width=100)
    before = torch.rand(60, heads[1], 1600, device="cuda")
    got = TC.check_weights(q, cache, table, k, lens, counts, lse, causal=causal, before=before, decay=0.75)
    assert torch.equal(ha.cache_weights(q, cache, table, CU.ints(lens), lse, CU.offsets(counts), weights=before, decay=0.75, causal=causal, out=before), got)
    again = ha.cache_chunk_attention(q, cache, table, CU.ints(lens), CU.offsets(counts), causal=causal)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("heads,many", [((2, 2, 64), 60), ((4, 1, 128), 60), ((2, 1, 64), 17), ((32, 8, 128), 16)])
def test_large_parts_beside_single_tokens(heads, many):
    """More rows a request on average than the few rows' kernels take a request, and requests that suit them all the same."""
    lens, counts = [33 + 19 * i for i in range(many)], [1] * many
    for r, n in ((1, 700), (2, 3), (many // 2, 1900), (many - 1, 260)):
        counts[r], lens[r] = n, max(lens[r], n // 2 + 300)
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, heads, 64, torch.float16)
    before = torch.rand(many, heads[1], table.shape[1] * 64, device="cuda")
    TC.check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.75)


@pytest.mark.parametrize("heads", [260, 40, 20])
def test_one_token_of_very_many_heads(heads):
    lens = [1 + 37 * i for i in range(17)]
    cache, table, k, v = CU.filled(lens, 1, 64, 16)
    q = TC.queries(17, heads, 64, torch.bfloat16)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints(lens))
    CU.check_attention((out, lse), CU.attention(q.double(), k, v, lens, [1] * 17), torch.bfloat16, max(lens), 17)
    w = torch.rand(17, 1, table.shape[1] * 16, device="cuda")
    want, bound = CU.weights(q.double(), k, lens, [1] * 17, lse, w, 0.5, cap=w.shape[2])
    got = ha.cache_weights(q, cache, table, CU.ints(lens), lse, weights=w, decay=0.5, out=w)
    assert bool(((got.double() - want).abs() <= bound).all())
