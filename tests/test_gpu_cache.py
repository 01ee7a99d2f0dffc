"""The paged 4-bit cache: scheduling, storing, reading and attention of one token, against plain statements of the operators."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
import serving_util as SU

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---- plan -------------------------------------------------------------------------------------------------------------------
def _step(rng, R, W, page, spare, end=0.2, prompt=0):
    lens = rng.integers(0, W * page + 1, R)
    kind = rng.random(R)
    new = np.where(kind < end, -1, np.where(kind < 0.5, rng.integers(0, 3, R), rng.integers(0, prompt + 1, R)))
    need = -(-lens // page)
    order = rng.permutation(int(need.sum()) + spare + 5)
    table = np.full((R, W), -1)
    at = 0
    for r in range(R):
        table[r, :need[r]] = order[at:at + need[r]]
        at += need[r]
    free = np.full(len(order), -1)
    free[:spare] = order[at:at + spare]
    return lens, new, table, free, spare


@pytest.mark.parametrize("R,W,page,spare,prompt,rows", [
    (1, 1, 16, 1, 1, 4), (1, 7, 64, 0, 5, 9), (5, 8, 16, 6, 40, 50), (40, 13, 48, 30, 100, 700), (40, 12, 16, 0, 60, 100),
    (513, 4, 32, 300, 90, 20000), (1000, 33, 64, 100000, 10, 3000), (4096, 3, 16, 900, 5, 9000)])
def test_plan(R, W, page, spare, prompt, rows):
    rng = np.random.default_rng(R * 1000 + W)
    for _ in range(3):
        lens, new, table, free, n_free = _step(rng, R, W, page, spare, prompt=prompt)
        want = SU.plan(lens, new, table.tolist(), free, n_free, page, rows)
        before = [ints(x) for x in (lens, new, table, free, [n_free])]
        given = [x.clone() for x in before]
        got = ha.cache_plan(*given, page, rows)
        for name, x in got._asdict().items():
            assert np.array_equal(x.cpu().numpy(), np.asarray(want[name])), name
        assert all(torch.equal(a, b) for a, b in zip(before, given))          # the inputs are as they were


def test_plan_steps_follow_each_other():
    """Requests come, grow and end over many steps; no page is ever had twice or lost."""
    rng = np.random.default_rng(3)
    R, W, page, pages = 9, 6, 16, 30
    state = [ints(np.zeros(R)), ints(np.full((R, W), -1)), ints(rng.permutation(pages)), ints([pages])]
    for step in range(60):
        lens = state[0].cpu().numpy()
        new = np.where(rng.random(R) < 0.15, -1, rng.integers(0, 20, R))
        got = ha.cache_plan(state[0], ints(new), state[1], state[2], state[3], page, 200)
        want = SU.plan(lens, new, state[1].cpu().numpy().tolist(), state[2].cpu().numpy(), int(state[3]), page, 200)
        for name, x in got._asdict().items():
            assert np.array_equal(x.cpu().numpy(), np.asarray(want[name])), (step, name)
        owned = got.table.cpu().numpy().ravel().tolist() + got.free.cpu().numpy()[:int(got.n_free)].tolist()
        assert sorted(x for x in owned if x >= 0) == list(range(pages))
        state = [got.lengths, got.table, got.free, got.n_free]


def test_plan_takes_odd_numbers():
    """Lengths below zero count as zero, a request longer than its table keeps what the table holds, no requests are no work."""
    got = ha.cache_plan(ints([-5, 100]), ints([3, 2]), ints([[-1, -1], [4, 9]]), ints([1, 2, 3]), ints([2]), 16, 6)
    assert got.table.cpu().tolist() == [[2, -1], [4, 9]] and got.lengths.cpu().tolist() == [3, 100]
    assert got.slots.cpu().tolist() == [32, 33, 34, -1, -1, -1]
    got = ha.cache_plan(ints([]), ints([]), ints(np.zeros((0, 4))), ints([1, 2]), ints([2]), 16, 3)
    assert got.slots.cpu().tolist() == [-1] * 3 and got.cu_new.cpu().tolist() == [0] and got.free.cpu().tolist() == [1, 2]


# ---- store and read ---------------------------------------------------------------------------------------------------------
def _values(kind, rng, shape, dtype):
    x = rng.standard_normal(shape)
    if kind == "offset":
        x = x + 5 * rng.standard_normal(shape[1:])
    elif kind == "wide":
        x = x * 10.0 ** rng.integers(-6, 4, shape[:-1] + (1,))
    elif kind == "coarse":
        x = np.round(x * 2) / 2                       # many ties, many constant groups
        x[::3] = 1.5
        x[1::5] = 0
    elif kind == "broken":
        x[0, 0, 3], x[1, 0, 40], x[2, 0, 0], x[3, 0, 33] = np.inf, -np.inf, np.nan, 3e38
        x[4] = 7e4
    return torch.tensor(x, dtype=torch.float32).to(dtype).cuda()


@pytest.mark.parametrize("kind", ["normal", "offset", "wide", "coarse", "broken"])
@pytest.mark.parametrize("heads,d,page,dtype", [(3, 64, 16, "bf16"), (1, 128, 64, "fp16"), (4, 128, 48, "bf16"), (2, 64, 128, "fp16")])
def test_store_and_read(kind, heads, d, page, dtype):
    rng = np.random.default_rng(len(kind) + d)
    lens = [1, page - 1, page, page + 1, 0, 2 * page + 17, 3]
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + 2)
    table = np.full((len(lens), max(need)), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    slots = np.concatenate([[table[r, t // page] * page + t % page for t in range(n)] for r, n in enumerate(lens)]).astype(int)
    T = len(slots)
    k, v = (_values(kind, rng, (T, heads, d), DT[dtype]) for _ in range(2))
    cache = ha.cache_pages(len(order), heads, d, page)
    ha.cache_store(cache, k, v, ints(slots))
    cu = ints(np.concatenate([[0], np.cumsum(lens)]))
    want = [SU.held(x.float().cpu().numpy()) for x in (k, v)]
    got = ha.cache_read(cache, ints(table), cu, T, dtype=torch.float32)
    for w, g in zip(want, got):
        assert np.array_equal(g.cpu().numpy(), w, equal_nan=True)
    for t in (torch.bfloat16, torch.float16):
        for w, g in zip(want, ha.cache_read(cache, ints(table), cu, T, dtype=t)):
            assert torch.equal(g.cpu().nan_to_num(nan=77.0), torch.tensor(w).to(t).nan_to_num(nan=77.0))
    # the bytes are in the order that is written down: every whole block of the longest request
    r = int(np.argmax(lens))
    for b in range(lens[r] // 16):
        rows = slice(sum(lens[:r]) + 16 * b, sum(lens[:r]) + 16 * b + 16)
        block = cache[table[r, 16 * b // page], 0, 16 * b % page // 16].cpu().numpy()
        want_bytes = SU.block_bytes(k[rows, 0].float().cpu().numpy(), v[rows, 0].float().cpu().numpy())
        if kind == "broken":                          # NaNs may differ in their bits
            block, want_bytes = block[:16 * d], want_bytes[:16 * d]
        assert np.array_equal(block, want_bytes)


def test_store_with_every_scale():
    # groups from -7 s to 8 s with numbers at and beside the ties, for every s of fp16 with finite ends: the codes are those of the divisions
    rng = np.random.default_rng(5)
    s = np.arange(1, 0x7c00, dtype=np.uint16).view(np.float16).astype(np.float64)
    s = s[8 * s < 65504]
    s = s[:len(s) // 4 * 4]
    x = np.concatenate([s[:, None] * [[-7, 8]], s[:, None] * (rng.integers(-14, 17, (len(s), 30)) / 2)], 1)
    x = rng.permuted(x, axis=1).astype(np.float16).reshape(-1, 1, 64)
    for dtype in (torch.float16, torch.bfloat16):
        k, v = torch.tensor(x[0::2]).to(dtype).cuda(), torch.tensor(x[1::2]).to(dtype).cuda()
        T = len(k)
        cache = ha.cache_pages(-(-T // 64), 1, 64, 64)
        ha.cache_store(cache, k, v, ints(np.arange(T)))
        got = ha.cache_read(cache, ints(np.arange(len(cache))[None]), ints([0, T]), T, dtype=torch.float32)
        for w, g in zip((k, v), got):
            assert np.array_equal(g.cpu().numpy(), SU.held(w.float().cpu().numpy()))


def test_store_leaves_out_slots_that_are_none_and_touches_nothing_else():
    rng = np.random.default_rng(1)
    for d in (64, 128):
        cache = ha.cache_pages(4, 2, d, 32)
        cache.copy_(torch.randint(0, 255, cache.shape, dtype=torch.uint8))
        before = cache.clone()
        k = torch.randn(5, 2, d, device="cuda", dtype=torch.bfloat16)
        ha.cache_store(cache, k, k, ints([-1, 37, 4 * 32, 2 ** 31 - 1, 39]))
        changed = (cache != before).nonzero().cpu()
        assert set(changed[:, 0].tolist()) == {1} and set(changed[:, 2].tolist()) == {0}
        ha.cache_store(cache, k[:0], k[:0], ints([]))
        got = ha.cache_read(cache, ints([[1]]), ints([0, 8]), 8, dtype=torch.float32)[0]
        want = SU.held(k.float().cpu().numpy())
        assert np.array_equal(got[5].cpu().numpy(), want[1]) and np.array_equal(got[7].cpu().numpy(), want[4])
        # the tokens beside them are as they were
        kept = ha.cache_read(before, ints([[1]]), ints([0, 8]), 8, dtype=torch.float32)[0]
        for t in (0, 1, 2, 3, 4, 6):
            assert torch.equal(got[t].nan_to_num(), kept[t].nan_to_num())


def test_strides_and_windows():
    """Rows that are views of a larger tensor, in another order of its axes too; a window of a request's tokens; rows without a place."""
    rng = np.random.default_rng(2)
    T, H, d = 50, 3, 64
    for layout in range(3):
        if layout == 0:
            qkv = torch.randn(T, 3 * H, d, device="cuda").bfloat16()
            k, v = qkv[:, H:2 * H], qkv[:, 2 * H:]
        elif layout == 1:
            k, v = (torch.randn(H, T, d, device="cuda").bfloat16().transpose(0, 1) for _ in range(2))
        else:
            k, v = (torch.randn(T, H, d + 1, device="cuda").bfloat16()[:, :, 1:] for _ in range(2))      # copied by the binding
        cache = ha.cache_pages(3, H, d, 32)
        order = [2, 0]
        ha.cache_store(cache, k, v, ints([order[t // 32] * 32 + t % 32 for t in range(T)]))
        want = [SU.held(x.float().cpu().numpy()) for x in (k, v)]
        got = ha.cache_read(cache, ints([order, [-1, 1]]), ints([0, 20, 25]), 30, first=ints([17, 30]), dtype=torch.float32)
        for w, g in zip(want, got):
            g = g.cpu().numpy()
            assert np.array_equal(g[:20], w[17:37]) and not g[20:].any()
        got = ha.cache_read(cache, ints([order]), ints([0, 90]), 90, dtype=torch.float32)                  # beyond the table: zeros
        assert not got[0][64:].any()
        got = ha.cache_read(cache, ints([order]), ints([0, 9]), 9, first=ints([-4]), dtype=torch.float32)  # before the first token: zeros
        assert not got[1][:4].any() and np.array_equal(got[1][4:].cpu().numpy(), want[1][:5])


# ---- attention of one token ---------------------------------------------------------------------------------------------------
def _context(rng, lens, heads, d, page, dtype, scale=1.0, spare=3):
    need = [-(-n // page) for n in lens]
    order = rng.permutation(sum(need) + spare)
    table = np.full((len(lens), max(max(need), 1) + 1), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    # what no token has written may hold anything: NaN scales among it
    cache = torch.full((len(order), heads, page // 16, 20 * d), 0xff, dtype=torch.uint8, device="cuda")
    T = sum(lens)
    k = torch.tensor(scale * (rng.standard_normal((T, heads, d)) + rng.standard_normal((heads, d)))).to(DT[dtype]).cuda()
    v = torch.tensor(rng.standard_normal((T, heads, d))).to(DT[dtype]).cuda()
    slots = [table[r, t // page] * page + t % page for r, n in enumerate(lens) for t in range(n)]
    if T:
        ha.cache_store(cache, k, v, ints(slots))
    return cache, table, SU.held(k.float().cpu().numpy()).astype(np.float64), SU.held(v.float().cpu().numpy()).astype(np.float64)


def _check(q, lens, K, V, out, lse, scale=None, skip=None):
    """out, lse (fp32) against 64 bits.  Weights and values enter as fp16 (2^-11 each, the sum of weights with the first), the scores are sums of
    at most 128 products and a handful of terms 64 times as large in fp32 (2^-16 of sum |q k|), exp2 and the sums take a few 2^-22."""
    R, H, d = q.shape
    G = H // K.shape[1]
    at = 0
    for r, n in enumerate(lens):
        keep = np.ones(n, bool) if skip is None else ~np.asarray(skip(r, np.arange(n)), bool)
        for h in range(H):
            k, v = K[at:at + n, h // G][keep], V[at:at + n, h // G][keep]
            o, l, mass, size = SU.attention(SU.f64(q[r, h:h + 1]), k, v, [len(k)], scale)
            err = 2.0 ** -16 * size[0]
            assert np.all(np.abs(out[r, h] - o[0]) <= (2 * 2.0 ** -11 + 2 * err + 1e-5) * mass[0] + 1e-6), (r, h)
            if n and len(k):
                assert abs(lse[r, h] - l[0]) <= err + 2.0 ** -21 * abs(l[0]) + 2e-6, (r, h)
            else:
                assert lse[r, h] == -np.inf and not out[r, h].any()
        at += n


@pytest.mark.parametrize("hq,hkv,d,page,dtype", [(4, 4, 64, 16, "fp16"), (4, 1, 128, 64, "bf16"), (9, 3, 64, 32, "bf16"), (8, 1, 128, 16, "fp16"), (28, 4, 128, 64, "fp16"),
                                                 (9, 1, 64, 128, "bf16"), (32, 2, 128, 64, "bf16"), (20, 1, 128, 48, "bf16"), (40, 1, 64, 64, "fp16")])
def test_cache_attention(hq, hkv, d, page, dtype):
    rng = np.random.default_rng(hq * d + page)
    lens = [0, 1, 2, 15, 16, 17, page - 1, page, page + 1, 3 * page + 5, 700, 0, 1203]
    cache, table, K, V = _context(rng, lens, hkv, d, page, dtype)
    q = torch.tensor(rng.standard_normal((len(lens), hq, d))).to(DT[dtype]).cuda()
    out, lse = ha.cache_attention(q, cache, ints(table), ints(lens), out_dtype=torch.float32)
    _check(q, lens, K, V, out.cpu().numpy(), lse.cpu().numpy())
    short, lse2 = ha.cache_attention(q, cache, ints(table), ints(lens))
    assert torch.equal(short, out.to(DT[dtype])) and torch.equal(lse, lse2)


def test_cache_attention_long_contexts_and_few_requests():
    rng = np.random.default_rng(7)
    for lens, hq, hkv, d in (([20011], 4, 1, 128), ([9000, 1, 33], 2, 2, 64), ([5000] * 3, 32, 2, 64)):
        cache, table, K, V = _context(rng, lens, hkv, d, 64, "bf16")
        q = torch.tensor(rng.standard_normal((len(lens), hq, d))).to(torch.bfloat16).cuda()
        out, lse = ha.cache_attention(q, cache, ints(table), ints(lens), out_dtype=torch.float32)
        _check(q, lens, K, V, out.cpu().numpy(), lse.cpu().numpy())


@pytest.mark.parametrize("size", [1.0, 0.002, 50.0, 5000.0])
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
def test_cache_attention_of_a_long_context_relative_to_its_result(d, dtype, size):
    """A result over 100000 tokens is a few hundred times smaller than what it is summed from (scales times codes, and minima): errors are held to
    the result.  Weights rounded to fp16 (bf16 queries) are 2^-11 each, independent of each other; everything else has to stay below that."""
    gen = torch.Generator("cuda").manual_seed(3)
    T, H, page = 100_003, 2, 64
    pages = -(-T // page)
    cache = ha.cache_pages(pages, H, d, page)
    k, v = (torch.randn(T, H, d, generator=gen, device="cuda").to(DT[dtype]) for _ in range(2))
    v = (v.float() * size).to(DT[dtype])
    q = torch.randn(1, 2 * H, d, generator=gen, device="cuda").to(DT[dtype])
    ha.cache_store(cache, k, v, torch.arange(T, dtype=torch.int32, device="cuda"))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    K, V = (x.double() for x in ha.cache_read(cache, table, ints([0, T]), T, dtype=torch.float32))
    out, _ = ha.cache_attention(q, cache, table, ints([T]), out_dtype=torch.float32)
    for h in range(2 * H):
        p = torch.softmax(K[:, h // 2] @ q[0, h].double() / d ** 0.5, 0)
        want = p @ V[:, h // 2]
        assert (out[0, h] - want).norm() <= 2.0 ** -11 * want.norm(), (h, float((out[0, h] - want).norm() / want.norm()))


def test_cache_attention_many_short_requests():
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 90, 777).tolist()
    cache, table, K, V = _context(rng, lens, 2, 64, 32, "fp16")
    q = torch.tensor(rng.standard_normal((len(lens), 6, 64))).half().cuda()
    out, lse = ha.cache_attention(q, cache, ints(table), ints(lens), out_dtype=torch.float32)
    _check(q, lens, K, V, out.cpu().numpy(), lse.cpu().numpy())


def test_cache_attention_scores_of_every_size():
    """Scores that grow along the context (the reference moves again and again), large and tiny queries, a scale of the caller's."""
    rng = np.random.default_rng(9)
    lens, d = [300, 2000], 128
    for dtype, qscale, scale in (("bf16", 1.0, 0.5), ("bf16", 1e-9, None), ("bf16", 1e6, 1e-6), ("fp16", 30.0, None), ("fp16", 1e-5, 3000.0)):
        cache, table, K, V = _context(rng, lens, 1, d, 64, dtype)
        k = torch.tensor(np.linspace(0.01, 6, sum(lens))[:, None, None] * np.ones((1, 1, d)) + 0.1 * rng.standard_normal((sum(lens), 1, d))).to(DT[dtype]).cuda()
        v = torch.tensor(rng.standard_normal((sum(lens), 1, d))).to(DT[dtype]).cuda()
        slots = [table[r, t // 64] * 64 + t % 64 for r, n in enumerate(lens) for t in range(n)]
        ha.cache_store(cache, k, v, ints(slots))
        K, V = (SU.held(x.float().cpu().numpy()).astype(np.float64) for x in (k, v))
        q = torch.tensor(qscale * np.abs(rng.standard_normal((2, 3, d)))).to(DT[dtype]).cuda()
        out, lse = ha.cache_attention(q, cache, ints(table), ints(lens), scale=scale or 0.0, out_dtype=torch.float32)
        _check(q, lens, K, V, out.cpu().numpy(), lse.cpu().numpy(), scale)


def test_cache_attention_pages_that_do_not_exist_hold_no_tokens():
    rng = np.random.default_rng(10)
    lens, page = [200, 64, 130], 32
    cache, table, K, V = _context(rng, lens, 2, 64, page, "bf16")
    table[0, 1], table[0, 3], table[1, 0], table[1, 1], table[2, 4] = -1, cache.shape[0], -1, -7, 2 ** 31 - 1
    gone = {0: {1, 3}, 1: {0, 1}, 2: {4}}
    q = torch.tensor(rng.standard_normal((3, 4, 64))).to(torch.bfloat16).cuda()
    out, lse = ha.cache_attention(q, cache, ints(table), ints(lens), out_dtype=torch.float32)
    _check(q, lens, K, V, out.cpu().numpy(), lse.cpu().numpy(), skip=lambda r, t: np.isin(t // page, list(gone[r])))
    # lengths below zero and beyond the table
    out, lse = ha.cache_attention(q, cache, ints(table), ints([-3, 0, 10 ** 9]), out_dtype=torch.float32)
    assert not out[:2].any() and torch.isinf(lse[:2]).all() and lse[2].isnan().any() == out[2].isnan().any()


def test_cache_attention_numbers_that_are_not_finite_stay_where_they_are():
    """NaN in a key reaches its request's heads, in a value that group's coordinates, in a query its own head: nothing else."""
    rng = np.random.default_rng(11)
    lens, d = [40, 77, 20], 64
    cache, table, K, V = _context(rng, lens, 2, d, 16, "bf16")
    q = torch.tensor(rng.standard_normal((3, 4, d))).to(torch.bfloat16).cuda()
    clean = ha.cache_attention(q, cache, ints(table), ints(lens), out_dtype=torch.float32)
    k1, v1 = (torch.ones(1, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k1[0, 0, 5] = float("nan")
    v1[0, 1, 40] = float("inf")
    ha.cache_store(cache, k1, v1, ints([table[1, 4] * 16 + 3]))                # token 67 of request 1
    q2 = q.clone()
    q2[2, 3, 1] = float("nan")
    out, lse = ha.cache_attention(q2, cache, ints(table), ints(lens), out_dtype=torch.float32)
    assert out[1, :2].isnan().all() and lse[1, :2].isnan().all()               # heads 0, 1 read key head 0
    assert out[1, 2:, 32:].isnan().all() and not out[1, 2:, :32].isnan().any() and not lse[1, 2:].isnan().any()
    assert out[2, 3].isnan().all()
    assert torch.equal(out[0], clean[0][0]) and torch.equal(out[2, :3], clean[0][2, :3])


def test_strided_queries_another_stream_and_a_graph():
    rng = np.random.default_rng(12)
    lens = [100, 31, 0, 514]
    cache, table, K, V = _context(rng, lens, 2, 128, 64, "bf16")
    wide = torch.randn(4, 12, 128, device="cuda").bfloat16()
    q = wide[:, 2:10]
    t, n = ints(table), ints(lens)
    want = ha.cache_attention(q.contiguous(), cache, t, n)
    got = ha.cache_attention(q, cache, t, n)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    got = ha.cache_attention(wide.transpose(0, 1).contiguous().transpose(0, 1)[:, 2:10], cache, t, n)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ha.cache_attention(q, cache, t, n)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    got = ha.cache_attention(q, cache, t, n, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # a captured decode step: lengths change between replays
    lengths, new = ints([100, 31, 0, 514]), ints([1, 1, 1, 1])
    free, n_free = ints([cache.shape[0] - 1]), ints([1])
    k = torch.randn(4, 2, 128, device="cuda").bfloat16()

    def step():
        plan = ha.cache_plan(lengths, new, t, free, n_free, 64, 4)
        ha.cache_store(cache, k, k, plan.slots)
        return (*ha.cache_attention(q, cache, plan.table, plan.lengths), plan.lengths)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = step()
    for start in ([100, 31, 0, 514], [90, 30, 1, 500]):
        lengths.copy_(ints(start))
        graph.replay()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
        assert held[2].cpu().tolist() == [x + 1 for x in start]


def test_offsets_beyond_32_bits():
    """A cache of more than 4 GB: its last page is written, read and attended to."""
    H, d, page = 32, 128, 64
    pages = (1 << 32) // (H * page // 16 * 20 * d) + 40
    cache = torch.zeros(pages, H, page // 16, 20 * d, dtype=torch.uint8, device="cuda")
    T = 70
    k, v = (torch.randn(T, H, d, device="cuda").bfloat16() for _ in range(2))
    table = [pages - 1, 1]
    ha.cache_store(cache, k, v, ints([table[t // page] * page + t % page for t in range(T)]))
    K, V = (SU.held(x.float().cpu().numpy()) for x in (k, v))
    got = ha.cache_read(cache, ints([table]), ints([0, T]), T, dtype=torch.float32)
    assert np.array_equal(got[0].cpu().numpy(), K) and np.array_equal(got[1].cpu().numpy(), V)
    q = torch.randn(1, H, d, device="cuda").bfloat16()
    out, lse = ha.cache_attention(q, cache, ints([table]), ints([T]), out_dtype=torch.float32)
    _check(q, [T], K.astype(np.float64), V.astype(np.float64), out.cpu().numpy(), lse.cpu().numpy())
    assert not cache[2:pages - 1].any()
