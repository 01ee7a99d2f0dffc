"""Cutting requests to the tokens of most weight, against plain statements: places, weights and every byte of what is moved."""
import math

import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU

pytestmark = pytest.mark.gpu


def some_weights(R, H, cap, seed=0, kind="tail"):
    gen = torch.Generator("cuda").manual_seed(seed)
    w = torch.randn(R, H, cap, generator=gen, device="cuda").mul(2).exp()
    if kind == "ties":
        w = torch.randint(0, 4, (R, H, cap), generator=gen, device="cuda").float()
    if kind == "zeros":
        w = torch.zeros(R, H, cap, device="cuda")
    if kind == "odd":                                   # no numbers, infinities, negative ones, both zeros, subnormal ones
        odd = torch.tensor([math.nan, math.inf, -math.inf, -1.0, 0.0, -0.0, 1e-42, 3e-45, 1.0], device="cuda")
        w = odd[torch.randint(0, 9, (R, H, cap), generator=gen, device="cuda")]
    return w


def check(lens, keep, heads, d, page, recent, first, kind="tail", dtype=torch.bfloat16, seed=0):
    room = sum(-(-n // page) for n in keep if n > 0)
    cache, table, k, v = CU.filled(lens, heads, d, page, dtype, seed, spare=room + 3)
    R, W = table.shape
    cap = W * page
    used = set(table.flatten().tolist())
    free = [p for p in range(cache.shape[0]) if p not in used]
    stack = CU.ints(free + [-1] * 4)
    plan = ha.cache_evict_plan(CU.ints(lens), CU.ints(keep), table, stack, CU.ints([len(free)]), page)
    want = CU.evict_plan(lens, keep, table.tolist(), stack.tolist(), len(free), page)
    for name, x in want.items():
        assert getattr(plan, name).tolist() == x, name
    w = some_weights(R, heads, cap, seed, kind)
    before = cache.clone()
    out, kept = ha.cache_evict(cache, w, table, CU.ints(lens), plan.table, plan.lengths, recent=recent, first=first)
    stay = CU.evict(w.cpu().numpy(), lens, plan.lengths.tolist(), recent, first)
    exp_w, exp_k = np.zeros((R, heads, cap), np.float32), np.full((R, heads, cap), -1, np.int32)
    wn = w.cpu().numpy()
    for r, n in enumerate(lens):
        if stay[r] is None:
            exp_w[r, :, :n] = wn[r, :, :n]
            continue
        for h in range(heads):
            exp_k[r, h, :len(stay[r][h])] = stay[r][h]
            exp_w[r, h, :len(stay[r][h])] = wn[r, h, stay[r][h]]
    assert np.array_equal(kept.cpu().numpy(), exp_k)
    assert np.array_equal(out.cpu().numpy().view(np.int32), exp_w.view(np.int32))
    # what the new pages stand for, number by number, and everything else as it was
    cu = CU.offsets(plan.lengths.tolist())
    rows = int(cu[-1])
    got_k, got_v = ha.cache_read(cache, plan.table, cu, rows, dtype=torch.float32)
    a = b = 0
    for r, n in enumerate(lens):
        m = int(plan.lengths[r])
        for h in range(heads):
            at = torch.tensor(stay[r][h] if stay[r] else list(range(m)), device="cuda", dtype=torch.long)
            for got, held in ((got_k, k), (got_v, v)):
                x, y = got[b:b + m, h], held[a:a + n, h][at].float()
                assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x.nan_to_num(), y.nan_to_num())
        a += n
        b += m
    new = sorted(set(plan.table.flatten().tolist()) - used - {-1})
    others = [p for p in range(cache.shape[0]) if p not in new]
    assert torch.equal(cache[others], before[others])
    return cache, plan, out, kept


@pytest.mark.parametrize("kind", ["tail", "ties", "zeros", "odd"])
@pytest.mark.parametrize("heads,d,page", [(2, 128, 64), (3, 64, 16), (1, 64, 128)])
def test_cuts(heads, d, page, kind):
    lens = [300, 17, 0, 1, 129, 1000, 64, 33, 500]
    keep = [100, 16, 5, 0, 128, 37, 64, -1, 499]
    check(lens, keep, heads, d, page, recent=10, first=4, kind=kind)


@pytest.mark.parametrize("recent,first", [(0, 0), (1, 0), (0, 7), (200, 3), (49, 1), (50, 1 << 20), (1 << 20, 1 << 20)])
def test_what_stays_in_any_case(recent, first):
    check([300, 51, 60], [50, 50, 1], 2, 64, 16, recent, first)


@pytest.mark.parametrize("lens,keep", [([4096], [4095]), ([4097, 8193], [4096, 1]), ([20000, 3], [777, 2]), ([131072], [9000]), ([65, 70001], [64, 70000])])
def test_long_contexts(lens, keep):
    check(lens, keep, 2, 64, 64, recent=100, first=4)
    check(lens, keep, 1, 128, 16, recent=0, first=0, kind="ties", dtype=torch.float16)


def test_groups_that_are_not_numbers_move_as_they_are():
    lens, keep = [200], [150]
    cache, table, k, v = CU.filled(lens, 2, 64, 16, torch.float16, spare=20, put=lambda k, v: (k[30].fill_(math.nan), v[77, 0, :5].fill_(math.inf)))
    used = set(table.flatten().tolist())
    free = [p for p in range(cache.shape[0]) if p not in used]
    plan = ha.cache_evict_plan(CU.ints(lens), CU.ints(keep), table, CU.ints(free), CU.ints([len(free)]), 16)
    w = some_weights(1, 2, table.shape[1] * 16)
    w[:, :, [30, 77]] = 1e9
    out, kept = ha.cache_evict(cache, w, table, CU.ints(lens), plan.table, plan.lengths)
    got = ha.cache_read(cache, plan.table, CU.offsets(keep), 150, dtype=torch.float32)
    for h in range(2):
        at = kept[0, h, :150].long()
        for x, y in zip(got, (k, v)):
            y = y[at, h].float()
            assert torch.equal(torch.isnan(x[:, h]), torch.isnan(y)) and torch.equal(x[:, h].nan_to_num(), y.nan_to_num())


def test_missing_pages():
    """Tokens in a page that is none are zeros; a new page that is none is not written."""
    lens, keep = [100], [60]
    cache, table, k, v = CU.filled(lens, 1, 64, 16, spare=20)
    used = set(table.flatten().tolist())
    free = [p for p in range(cache.shape[0]) if p not in used]
    plan = ha.cache_evict_plan(CU.ints(lens), CU.ints(keep), table, CU.ints(free), CU.ints([len(free)]), 16)
    table[0, 1], to = -1, plan.table.clone()
    to[0, 2] = -1
    before = cache.clone()
    w = some_weights(1, 1, table.shape[1] * 16)
    out, kept = ha.cache_evict(cache, w, table, CU.ints(lens), to, plan.lengths)
    got, _ = ha.cache_read(cache, to, CU.offsets(keep), 60, dtype=torch.float32)
    for i, t in enumerate(kept[0, 0, :60].tolist()):
        want = torch.zeros(64, device="cuda") if 16 <= t < 32 or 32 <= i < 48 else k[t, 0].float()
        assert torch.equal(got[i, 0], want), (i, t)
    written = [int(p) for p in to[0] if p >= 0]
    others = [p for p in range(cache.shape[0]) if p not in written]
    assert torch.equal(cache[others], before[others])


@pytest.mark.parametrize("R", [1, 7, 300, 4096])
def test_plans(R):
    rng = np.random.default_rng(R)
    W, page = 9, 16
    for share in (0.0, 0.3, 1.0):
        lens = rng.integers(0, W * page + 1, R)
        keep = np.where(rng.random(R) < 0.3, rng.integers(-3, 2, R), rng.integers(0, W * page + 20, R))
        need = -(-lens // page)
        pages = int(need.sum()) + R * W
        order = rng.permutation(pages)
        table = np.full((R, W), -1)
        table[np.arange(W)[None] < need[:, None]] = order[:need.sum()]
        n_free = int(share * R * W)
        free = np.full(pages, -1)
        free[:n_free] = order[need.sum():need.sum() + n_free]
        args = [CU.ints(x.tolist()) for x in (lens, keep, table, free)]
        got = ha.cache_evict_plan(*args, CU.ints([n_free]), page)
        for name, x in CU.evict_plan(lens.tolist(), keep.tolist(), table.tolist(), free.tolist(), n_free, page).items():
            assert getattr(got, name).tolist() == x, name
        # the same pages as before, each once
        all_pages = sorted(p for p in got.table.flatten().tolist() + got.free.tolist() if p >= 0)
        assert all_pages == sorted(p for p in table.flatten().tolist() + free.tolist() if p >= 0)


def test_no_requests():
    cache, table, k, v = CU.filled([20], 2, 64, 16)
    plan = ha.cache_evict_plan(CU.ints([]), CU.ints([]), table[:0], CU.ints([3, 4, -1]), CU.ints([2]), 16)
    assert plan.free.tolist() == [3, 4, -1] and plan.n_free.tolist() == [2] and plan.lengths.shape == (0,)
    w, kept = ha.cache_evict(cache, torch.zeros(0, 2, table.shape[1] * 16, device="cuda"), table[:0], CU.ints([]), table[:0], CU.ints([]))
    assert w.shape == kept.shape == (0, 2, table.shape[1] * 16)


def test_other_streams_and_graphs():
    lens, keep = [300, 90], [100, 90]
    cache, table, k, v = CU.filled(lens, 2, 64, 16, spare=30)
    used = set(table.flatten().tolist())
    free = [p for p in range(cache.shape[0]) if p not in used]
    w = some_weights(2, 2, table.shape[1] * 16)
    args = CU.ints(lens), CU.ints(keep), table, CU.ints(free), CU.ints([len(free)])
    plan = ha.cache_evict_plan(*args, 16)
    want = ha.cache_evict(cache, w, table, args[0], plan.table, plan.lengths, 5, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    p2 = ha.cache_evict_plan(*args, 16, stream=side.cuda_stream)
    got = ha.cache_evict(cache, w, table, args[0], p2.table, p2.lengths, 5, 5, stream=side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(torch.equal(x, y) for x, y in zip(plan, p2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p3 = ha.cache_evict_plan(*args, 16)
        got = ha.cache_evict(cache, w, table, args[0], p3.table, p3.lengths, 5, 5)
    for seed in (1, 2):
        w.copy_(some_weights(2, 2, table.shape[1] * 16, seed))
        graph.replay()
        again = ha.cache_evict(cache, w, table, args[0], plan.table, plan.lengths, 5, 5)
        assert all(torch.equal(x, y) for x, y in zip(got, again))
