"""The paged 4-bit cache where numbers come near the ends of their types."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("d,dtype,heads", [(64, "fp16", 1), (64, "bf16", 8), (128, "bf16", 4), (128, "fp16", 16)])
@pytest.mark.parametrize("size", [8.0, 300.0])
@pytest.mark.parametrize("nan", [False, True])
def test_values_of_several_scales_under_small_weights(d, dtype, heads, size, nan):
    """One token 16.5 octaves above 30 others that are alike and have all the values, in groups whose scales are on either side of powers of two (and with a
    NaN among them, which its own group alone shows).  Weights are fp16 numbers, 2^-11 off at most where they are not smaller than 2^-14: the largest is
    2^12 over the power of two in the scales of a block - 2^12 / 2^7 for values of 300 - and the others 2^-16.5 of that, 2^-11.5."""
    R, T, page = 50, 31, 32                              # (a request is less than what one warp takes: all its tokens meet)
    gen = torch.Generator("cuda").manual_seed(d + heads)
    cache = ha.cache_pages(R, 1, d, page)
    k = torch.zeros(R, T, 1, d, device="cuda")
    k[:, 7] = 16.5 * np.log(2) / (4 * d ** 0.5)
    v = size * (1 + torch.randn(R, T, 1, d, generator=gen, device="cuda") * torch.rand(R, T, 1, 1, generator=gen, device="cuda"))
    v[:, 7] = 0
    if nan:
        v[:, 20, 0, 40] = float("nan")
    k, v = (x.reshape(R * T, 1, d).to(DT[dtype]) for x in (k, v))
    ha.cache_store(cache, k, v, ints((np.arange(R)[:, None] * page + np.arange(T)).ravel()))
    table = ints(np.arange(R))[:, None]
    K, V = (x.view(R, T, d).double() for x in ha.cache_read(cache, table, ints(np.arange(R + 1) * T), R * T, dtype=torch.float32))
    q = torch.full((R, heads, d), 4.0, device="cuda").to(DT[dtype])
    out, lse = ha.cache_attention(q, cache, table, ints([T] * R), out_dtype=torch.float32)
    z = K @ q[0, 0].double() / d ** 0.5
    want = torch.einsum("rt,rtd->rd", torch.softmax(z, 1), V)[:, None]
    size_of = torch.einsum("rt,rtd->rd", torch.softmax(z, 1), V.abs())[:, None]
    bad = torch.zeros(d, dtype=torch.bool, device="cuda")
    if nan:
        bad[32:64] = True
    assert torch.equal(want.isnan(), bad.expand_as(want)) and out[:, :, bad].isnan().all()
    bound = (2.0 ** -11 + 2.0 ** -15 * float(z.max()) + 1e-5) * size_of
    assert ((out.double() - want).abs() <= bound)[:, :, ~bad].all(), float(((out.double() - want).abs() / size_of)[:, :, ~bad].max())
    assert (lse.double() - torch.logsumexp(z, 1)[:, None]).abs().max() <= 1e-4


def test_a_plan_of_more_new_tokens_than_an_int_counts():
    """Requests that bring 2^31 - 1 tokens have no room and are not admitted; their tokens count, up to 2^31 - 1, and push the others' out of the batch."""
    most = 2 ** 31 - 1
    for R, at in ((6, 0), (600, 500)):                   # (in one thread's share, and far behind others)
        lens, new, table = np.zeros(R, np.int64), np.zeros(R, np.int64), np.full((R, 4), -1)
        lens[at:at + 6], new[at:at + 6] = [3, 0, 40, 1, most, most], [5, most, 7, most, 2, -1]
        table[at, 0], table[at + 2, :3], table[at + 3, 0], table[at + 4], table[at + 5] = 0, [1, 2, 3], 4, [5, 6, 7, 8], [9, 10, 11, 12]
        free = np.concatenate([np.arange(20, 30), [-1] * 6])
        got = ha.cache_plan(ints(lens), ints(new), ints(table), ints(free), ints([10]), 16, 12)
        assert got.slots.cpu().tolist() == [3, 4, 5, 6, 7] + [-1] * 7 and got.positions.cpu().tolist() == [3, 4, 5, 6, 7] + [-1] * 7
        assert got.cu_new.cpu().tolist()[at:at + 7] == [0, 5] + [most] * 5 and got.cu_new.cpu().tolist()[-1] == most
        assert got.lengths.cpu().tolist()[at:at + 6] == [8, 0, 47, 1, most, 0]
        assert got.cu_len.cpu().tolist()[at:at + 7] == [0, 8, 8, 55, 56, most, most]
        want = table.copy()
        want[at + 5] = -1
        assert np.array_equal(got.table.cpu().numpy(), want)          # (47 tokens fit the three pages that there were)
        assert int(got.n_free) == 14 and got.free.cpu().tolist() == [*range(20, 30), 9, 10, 11, 12, -1, -1]


def test_attention_of_a_length_that_fills_the_longest_table():
    """2^31 - 16 tokens, of which 200 exist: the other pages of the table do not."""
    gen = torch.Generator("cuda").manual_seed(1)
    for d, dtype in ((64, "fp16"), (128, "bf16")):
        cache = ha.cache_pages(20, 1, d, 16)
        k, v = (torch.randn(200, 1, d, generator=gen, device="cuda").to(DT[dtype]) for _ in range(2))
        ha.cache_store(cache, k, v, ints(np.arange(200)))
        width = (1 << 27) - 1
        table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
        table[0, :6], table[0, -7:-1] = ints(np.arange(6)), ints(np.arange(6, 12))
        q = torch.randn(1, 2, d, generator=gen, device="cuda").to(DT[dtype])
        want = ha.cache_attention(q, cache, ints(np.arange(12))[None], ints([192]), out_dtype=torch.float32)
        got = ha.cache_attention(q, cache, table, ints([2 ** 31 - 1]), out_dtype=torch.float32)
        assert (got[0] - want[0]).abs().max() <= 2.0 ** -10 * want[0].abs().max() and (got[1] - want[1]).abs().max() <= 1e-5
        assert ha.last_device_status() == 0


def test_attention_of_nearly_as_many_units_as_an_int_counts():
    """64 heads over nearly 2^30 tokens, of which 70 exist, in the last page of the table."""
    gen = torch.Generator("cuda").manual_seed(2)
    d, heads, page, width = 128, 64, 1024, (1 << 20) - 1
    cache = ha.cache_pages(1, heads, d, page)
    k, v = (torch.randn(70, heads, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    ha.cache_store(cache, k, v, ints(np.arange(70)))
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0
    q = torch.randn(1, heads, d, generator=gen, device="cuda").bfloat16()
    want = ha.cache_attention(q, cache, ints([[0]]), ints([70]), out_dtype=torch.float32)
    got = ha.cache_attention(q, cache, table, ints([(width - 1) * page + 70]), out_dtype=torch.float32)
    assert (got[0] - want[0]).abs().max() <= 2.0 ** -10 * want[0].abs().max() and (got[1] - want[1]).abs().max() <= 1e-5
    assert ha.last_device_status() == 0


def test_a_plan_of_no_requests_says_what_one_of_idle_requests_says():
    for n_free in (-3, 0, 2, 9):
        free = ints([5, 6, 7, 8])
        got = ha.cache_plan(ints([]), ints([]), ints(np.zeros((0, 4))), free, ints([n_free]), 16, 3)
        want = ha.cache_plan(ints([0]), ints([0]), ints([[-1] * 4]), free, ints([n_free]), 16, 3)
        for name in ("slots", "positions", "free", "n_free"):
            assert torch.equal(getattr(got, name), getattr(want, name)), (n_free, name)
    for rows, page in ((-1, 16), (3, 0)):
        for R in (0, 2):
            with pytest.raises(ha.HyperAttnError):
                ha.cache_plan(ints([0] * R), ints([0] * R), ints(np.zeros((R, 4))), ints([1]), ints([1]), page, rows)
