"""Sums over long contexts: chunks of many rows whose segments have a CTA each, so that nothing but the kernels' own limit ends a chain of products."""
import math

import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU
import test_gpu_cache_chunk as TC

pytestmark = pytest.mark.gpu


def context(length, heads, d, dtype, change, page=64):
    """A cache of one request, its table, and K and V in 64 bits as it holds them.  change(k, v, first token): what is stored."""
    gen = torch.Generator("cuda").manual_seed(7)
    pages = -(-length // page)
    cache = ha.cache_pages(pages, heads, d, page)
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None].contiguous()
    for a in range(0, length, 8192):
        n = min(8192, length - a)
        k, v = (torch.randn(n, heads, d, generator=gen, device="cuda") for _ in range(2))
        k, v = change(k, v, a)
        token = torch.arange(a, a + n, device="cuda")
        ha.cache_store(cache, k.to(dtype), v.to(dtype), (table[0, token // page] * page + token % page).int())
    k, v = ha.cache_read(cache, table, CU.ints([0, length]), length, dtype=torch.float32)
    return cache, table, k.double(), v.double()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,rows,length", [((16, 16, 64), 2560, 65536), ((8, 8, 128), 5120, 40000), ((160, 160, 64), 100, 30001)])
def test_values_of_one_sign_do_not_drift(heads, rows, length, dtype):
    """The tensor cores cut some 1.2 2^-23 of the partial sum from every sum of 16 products, always downwards; values of one sign show what that comes to.  No chain is longer than 384 sums (fp16
    queries: 768, the weights' second part among them), so 512 (1024) times 2^-23, and the partial sum is half of the last one on average; roundings of weights, of values and of their sums differ in
    sign: 2^-11 over the root of the tokens that have weight (thousands) leave less than 1e-5.  (One chain over 65536 tokens: 3e-4.)"""
    cache, table, k, v = context(length, heads[1], heads[2], CU.TYPES[dtype], lambda k, v, a: (k, 1 + 0.2 * v))
    q = TC.queries(rows, heads[0], heads[2], CU.TYPES[dtype], scale=0.3)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints([length]), CU.offsets([rows]), out_dtype=torch.float32)
    pick = [0, 1, rows // 2, rows - 1]                             # (rows, of which every fourth head or so is looked at)
    hs = list(range(0, heads[0], max(1, heads[0] // 4)))
    seen = torch.arange(length, device="cuda") <= torch.tensor(pick, device="cuda")[:, None] + length - rows
    off = []
    for h in hs:
        z = (q[pick, h].double() @ k[:, h].T / math.sqrt(heads[2])).masked_fill(~seen, -math.inf)
        want = z.softmax(-1) @ v[:, h]
        off.append(((out[pick, h].double() - want) / want).mean())
        assert bool((torch.logsumexp(z, -1) - lse[pick, h]).abs().max() <= 2.0 ** -17 * (z.abs() * seen).nan_to_num(0).amax() + 2.0 ** -17)
    sums = 1024 if dtype == "fp16" else 512
    drift = float(torch.stack(off).mean().abs())
    assert drift <= sums / 2 * 2.0 ** -23 + 1e-5, drift


def test_bf16_results_do_not_drift_either():
    """Chains of 2048 sums at most (32768 tokens): 1.5e-4 by the rule above, beside what rounding to bf16 leaves.  Rows of one coordinate do not count as different samples of that: over 131072 tokens
    their results differ by 0.2 / 2^8.5 = 5e-4 of their size, less than half a step of 2^-8, and are mostly rounded to the same number.  So the mean is that of 16 heads x 64 coordinates, 1.7e-3 / 32 = 5.3e-5
    off; four times that are allowed.  (One chain over all tokens: 6e-4.)  Values are spread from one to two, as results near one number would all be rounded to it."""
    length, rows, heads, d = 131072, 2560, 16, 64
    size = 1 + torch.arange(heads * d, device="cuda").view(heads, d) * 0.6180339887 % 1
    cache, table, k, v = context(length, heads, d, torch.bfloat16, lambda k, v, a: (k, size * (1 + 0.2 * v)))
    q = TC.queries(rows, heads, d, torch.bfloat16, scale=0.3)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints([length]), CU.offsets([rows]))
    pick = torch.arange(0, rows, rows // 16, device="cuda")
    seen = torch.arange(length, device="cuda") <= pick[:, None] + length - rows
    off = []
    for h in range(heads):
        want = (q[pick, h].double() @ k[:, h].T / math.sqrt(d)).masked_fill(~seen, -math.inf).softmax(-1) @ v[:, h]
        off.append(((out[pick, h].double() - want) / want).mean())
    drift = float(torch.stack(off).mean().abs())
    assert drift <= 1.5e-4 + 4 * 1.7e-3 / 32, drift


@pytest.mark.parametrize("missing", [(0, 9500), (9000, 20000), (100, 23000), (0, 0)])
@pytest.mark.parametrize("heads,rows", [((16, 16, 64), 2500), ((4, 4, 128), 5000), ((150, 150, 64), 70)])
def test_pieces_in_a_row(heads, rows, missing):
    """Stretches without pages, so that rows see nothing in some pieces of their segment; a NaN early and late; values whose size changes."""
    length, page = 24000, 64

    def change(k, v, a):
        t = torch.arange(a, a + k.shape[0], device="cuda")[:, None, None]
        v = torch.where(t < 12000, v * 2.0 ** -12, v)
        v[((t == 3000) | (t == length - 40)).expand_as(v) & (torch.arange(v.shape[2], device="cuda") == 33)] = math.nan
        return torch.where(t % 5000 == 77, k * 3, k), v

    cache, table, k, v = context(length, heads[1], heads[2], torch.bfloat16, change, page)
    first, end = missing[0] // page, missing[1] // page
    table[0, first:end] = -1
    there = torch.ones(length, dtype=torch.bool, device="cuda")
    there[first * page:end * page] = False
    q = TC.queries(rows, heads[0], heads[2], torch.bfloat16)
    hs = [0, heads[0] - 1]
    got = ha.cache_chunk_attention(q, cache, table, CU.ints([length]), CU.offsets([rows]), out_dtype=torch.float32)
    want = CU.attention(q[:, hs].double(), k[:, hs], v[:, hs], [length], [rows], there=there)
    CU.check_attention((got[0][:, hs], got[1][:, hs]), want, torch.float32, length, rows)
    again = ha.cache_chunk_attention(q, cache, table, CU.ints([length]), CU.offsets([rows]), out_dtype=torch.float32)
    assert torch.equal(again[0].view(torch.int32), got[0].view(torch.int32)) and torch.equal(again[1], got[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,rows", [((4, 4, 64), 3), ((8, 2, 64), 2), ((6, 2, 64), 5), ((4, 1, 128), 1), ((8, 1, 128), 3), ((4, 4, 64), 90), ((2, 1, 128), 70), ((8, 2, 128), 150)])
def test_fp32_results_show_what_rounding_weights_loses(heads, rows, dtype):
    """Values that are fp16 numbers and that the cache holds as they are (steps of 1/8 from -1 on), so that nothing but weights is rounded on the way to an fp32 result.  Weights rounded to fp16 alone
    would leave 2e-4 of it (the root mean square of a rounding to fp16, as many signs as tokens).  In two parts they are 2^-22 off; what is left are the sums: up to 128 of products with values and 33 of
    scores, 1.2 2^-23 of partial sums each: 2e-5 of the result and 5e-6 in scores of size one.  Twice that is the bound."""
    length = 1000

    def change(k, v, a):
        v = (v.mul(4).round().clamp(-8, 7)) / 8
        groups = v.view(*v.shape[:2], -1, 32)
        groups[..., 0], groups[..., 1] = -1, 0.875
        return k, v

    cache, table, k, v = context(length, heads[1], heads[2], CU.TYPES[dtype], change)
    assert torch.equal(v.half().double(), v) and torch.equal((v * 8).round(), v * 8)
    q = TC.queries(rows, heads[0], heads[2], CU.TYPES[dtype], scale=0.5)
    out, lse = ha.cache_chunk_attention(q, cache, table, CU.ints([length]), CU.offsets([rows]), out_dtype=torch.float32)
    want = CU.attention(q.double(), k, v, [length], [rows])[0]
    off, want = ((x.unflatten(-1, (-1, 32))[..., 2:]) for x in (out.double() - want, want))        # (not the two that make the steps, whose results are sums of one sign)
    assert float(off.norm() / want.norm()) <= 5e-5, float(off.norm() / want.norm())
