"""Exact attention over packed prompts where numbers come near the ends of their types: scores far apart, values that nobody may see, rows beside others, infinities, long contexts."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
from test_gpu_prompt import DT, ROUND, check, inputs, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("octaves", [100, 150, 300, 400, 600])
def test_one_key_far_above_all_others(d, dtype, octaves):
    """A request a column of a key tile: one query, two tiles of keys, the one that decides in that column of the tile that is walked second."""
    gen = torch.Generator("cuda").manual_seed(octaves + d)
    n, nq, nk = 128, [1] * 128, [256] * 128
    k = 0.05 * torch.randn(n, 256, 1, d, generator=gen, device="cuda")
    v = torch.randn(n * 256, 1, d, generator=gen, device="cuda").to(DT[dtype])
    k[torch.arange(n), torch.arange(n)] = octaves * np.log(2) / (4 * d ** 0.5)         # times q = 4, d of them, 1 / sqrt(d)
    k = k.reshape(n * 256, 1, d).to(DT[dtype])
    q = torch.full((n, 1, d), 4.0, device="cuda").to(DT[dtype])
    out, lse = ha.prompt_attention(q, k, v, offsets(nq), offsets(nk), out_dtype=torch.float32)
    check(q, k, v, nq, nk, True, out, lse)


@pytest.mark.parametrize("d,dtype,most", [(64, "bf16", 3e38), (128, "bf16", 3e38), (64, "fp16", 65504.0), (128, "fp16", 65504.0)])
def test_finite_values_that_a_query_does_not_see_have_no_influence(d, dtype, most):
    """The largest number of the type in later values, from every column of a tile on: not a bit of the earlier rows changes."""
    n = [70, 300]
    q, k, v = inputs(d, n, n, 2, 1, d, dtype)
    clean, lse_clean = ha.prompt_attention(q, k, v, offsets(n), out_dtype=torch.float32)
    for first in range(100, 229):
        v2 = v.clone()
        v2[70 + first:] = most if first % 2 else -most
        out, lse = ha.prompt_attention(q, k, v2, offsets(n), out_dtype=torch.float32)
        assert torch.equal(out[:70 + first], clean[:70 + first]) and torch.equal(lse[:70 + first], lse_clean[:70 + first]), first


@pytest.mark.parametrize("d,dtype,most", [(64, "bf16", 3e38), (128, "bf16", 3e38), (64, "fp16", 65504.0), (128, "fp16", 65504.0)])
def test_values_of_keys_without_weight_have_no_influence(d, dtype, most):
    """Keys at minus infinity have a weight of zero, whatever finite number their value is."""
    q, k, v = inputs(d + 1, [256], [256], 1, 1, d, dtype)
    q = q.abs() + 0.1
    gone = [j for j in range(256) if j % 16 in (3, 14, 15)]
    k[gone] = -float("inf")
    want, lse_want = ha.prompt_attention(q, k, v, offsets([256]), out_dtype=torch.float32)
    v[gone] = most
    out, lse = ha.prompt_attention(q, k, v, offsets([256]), out_dtype=torch.float32)
    assert torch.isfinite(out).all() and torch.equal(out, want) and torch.equal(lse, lse_want)


@pytest.mark.parametrize("octaves", [15.3, 20.7, 25.2])
@pytest.mark.parametrize("d", [64, 128])
def test_fp16_weights_of_a_long_even_rest(d, octaves):
    """One key far above 32767 others that are alike, which have all the values: the result is the rest's.  A weight is an fp16 number that may be 2^-25 off
    where it is small, beside a largest one of 2^7: 2^-32 of the values that are summed; otherwise weights and their sum are 2^-12 off."""
    n = 32768
    gen = torch.Generator("cuda").manual_seed(d)
    for place in (n - 1, 5):
        k = torch.zeros(n, 1, d, device="cuda", dtype=torch.float16)
        k[place] = octaves * np.log(2) / (4 * d ** 0.5)
        v = (100 + torch.randn(n, 1, d, generator=gen, device="cuda")).half()
        v[place] = 0
        q = torch.full((1, 1, d), 4.0, device="cuda", dtype=torch.float16)
        out, lse = ha.prompt_attention(q, k, v, offsets([1]), offsets([n]), out_dtype=torch.float32)
        z = (k[:, 0].double() @ q[0, 0].double()) / d ** 0.5
        w = torch.softmax(z, 0)
        want = w @ v[:, 0].double()
        bound = (2 * ROUND["fp16"] + 2 ** -16 * float(z.max()) + 1e-5) * want + 2.0 ** -32 * (v[:, 0].double().sum(0))
        assert ((out[0, 0].double() - want).abs() <= bound).all(), (place, float(((out[0, 0].double() - want) / want).abs().max()))
        assert abs(float(lse[0, 0]) - float(torch.logsumexp(z, 0))) <= 2.0 ** -17 * float(z.max()) + 1e-5


@pytest.mark.parametrize("mean", [0.0, 1.0])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(2, 2, 64, "fp16"), (4, 1, 128, "bf16"), (2, 1, 128, "fp16"), (1, 1, 64, "bf16")])
def test_131072_keys_relative_to_the_result(hq, hkv, d, dtype, mean):
    """The context of the headline configuration.  A result over so many values is a few hundred times smaller than they are: errors are held to the result.
    Weights are rounded to the type, independently of each other, and once as a sum; O is one chain of 8 x 1024 products, and the tensor cores cut what
    they add (up to 2^-23 of O each): 2^-10 together."""
    n, past = 131072 + 77, 131072 - 123
    gen = torch.Generator("cuda").manual_seed(d + hq)
    q = torch.randn(200, hq, d, generator=gen, device="cuda").to(DT[dtype])
    k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda") for _ in range(2))
    k, v = k.to(DT[dtype]), (v + mean).to(DT[dtype])
    out, lse = ha.prompt_attention(q, k, v, offsets([200]), offsets([n]), out_dtype=torch.float32)
    assert past + 200 == n
    for i in (0, 1, 63, 128, 199):
        for h in range(hq):
            g = h // (hq // hkv)
            z = k[:past + i + 1, g].double() @ q[i, h].double() / d ** 0.5
            want = torch.softmax(z, 0) @ v[:past + i + 1, g].double()
            err = float((out[i, h].double() - want).norm() / want.norm())
            assert err <= 2 * ROUND[dtype] + 2.0 ** -10, (i, h, err)
            assert abs(float(lse[i, h]) - float(torch.logsumexp(z, 0))) <= 1e-4


def _seen_unfinite(v, n, causal):
    """For every row and coordinate of the packed prompts: has it seen +infinity or NaN, -infinity or NaN?"""
    up, down = ~(v < float("inf")), ~(v > -float("inf"))
    got, at = [], 0
    for a in n:
        for x in (up, down):
            x = x[at:at + a].int()
            got.append((x.cumsum(0) > 0) if causal else (x.sum(0, keepdim=True) > 0).expand_as(x))
        at += a
    return torch.cat(got[0::2]), torch.cat(got[1::2])


def _check_unfinite(v, n, causal, out, lse, clean, lse_clean):
    group = out.shape[1] // v.shape[1]
    up, down = (x.repeat_interleave(group, 1) for x in _seen_unfinite(v, n, causal))
    want = torch.where(up & down, float("nan"), torch.where(up, float("inf"), -float("inf")))
    bad = up | down
    assert torch.equal(out[bad].nan_to_num(nan=5.0, posinf=6.0, neginf=7.0), want[bad].nan_to_num(nan=5.0, posinf=6.0, neginf=7.0))
    assert torch.equal(out[~bad], clean[~bad]) and torch.equal(lse, lse_clean)
    assert ha.last_device_status() == 0


@pytest.mark.parametrize("d,G,dtype", [(64, 1, "bf16"), (64, 4, "fp16"), (128, 1, "fp16"), (128, 16, "bf16")])
@pytest.mark.parametrize("causal", [True, False])
def test_infinities_and_nan_reach_exactly_the_rows_that_see_them(d, G, dtype, causal):
    n = [300, 129, 1, 0, 40, 700]
    q, k, v = inputs(d + G, n, n, 2 * G, 2, d, dtype)
    clean, lse_clean = ha.prompt_attention(q, k, v, offsets(n), causal=causal, out_dtype=torch.float32)
    inf, nan = float("inf"), float("nan")
    for places in ([(299, 0, 5, nan)], [(0, 1, 0, inf)], [(130, 0, 9, inf), (250, 0, 9, -inf), (251, 1, 33, -inf), (127, 0, 63, nan)],
                   [(428, 0, 1, -inf), (429, 1, 2, inf), (469, 0, 3, nan), (470, 0, 3, inf)], [(470 + 127 * i, i % 2, 7 * i, (nan, inf, -inf)[i % 3]) for i in range(6)]):
        v2 = v.clone()
        for key, head, x, value in places:
            v2[key, head, x] = value
        _check_unfinite(v2, n, causal, *ha.prompt_attention(q, k, v2, offsets(n), causal=causal, out_dtype=torch.float32), clean, lse_clean)
    v2 = v.clone()
    v2[400:] = inf                                       # all of them, from somewhere on
    _check_unfinite(v2, n, causal, *ha.prompt_attention(q, k, v2, offsets(n), causal=causal, out_dtype=torch.float32), clean, lse_clean)


def test_infinities_in_many_prompts():
    rng = np.random.default_rng(12)
    n = rng.integers(0, 500, 150).tolist()
    q, k, v = inputs(12, n, n, 8, 2, 64, "bf16")
    clean, lse_clean = ha.prompt_attention(q, k, v, offsets(n), out_dtype=torch.float32)
    for share in (1e-6, 1e-5, 1e-4):
        v2 = torch.where(torch.tensor(rng.random(v.shape) < share, device="cuda"), float("inf"), v)
        _check_unfinite(v2, n, True, *ha.prompt_attention(q, k, v2, offsets(n), out_dtype=torch.float32), clean, lse_clean)


def test_a_query_that_only_sees_keys_at_minus_infinity_has_no_result_whatever_their_values():
    q, k, v = inputs(13, [200], [200], 1, 1, 64, "bf16")
    q = q.abs() + 0.1
    k[:150], v[:150] = -float("inf"), float("inf")
    out, lse = ha.prompt_attention(q, k, v, offsets([200]), out_dtype=torch.float32)
    assert not out[:150].any() and (lse[:150] == -float("inf")).all()


@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16")])
def test_one_bad_value_does_not_make_a_call_slow(d, dtype):
    """A value that every row sees, and one in each tile of keys.  (Four times as long as without: what the clock may do, and the rows that see them.)"""
    n = [6000]
    q, k, v = inputs(14, n, n, 2, 1, d, dtype)
    v2 = v.clone()
    v2[0, 0, 3], v2[100::128, 0, 7] = float("nan"), float("inf")
    cu = offsets(n)
    clean, lse_clean = ha.prompt_attention(q, k, v, cu, out_dtype=torch.float32)
    _check_unfinite(v2, n, True, *ha.prompt_attention(q, k, v2, cu, out_dtype=torch.float32), clean, lse_clean)

    def time(values):
        took = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                ha.prompt_attention(q, k, values, cu)
            b.record()
            b.synchronize()
            took.append(a.elapsed_time(b))
        return min(took)

    once = time(v)
    assert time(v2) <= 4 * once, (time(v2), once)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(6, 2, 64, "fp16"), (7, 1, 128, "fp16"), (5, 1, 64, "bf16"), (3, 3, 128, "bf16"), (24, 2, 64, "fp16")])
@pytest.mark.parametrize("causal", [True, False])
def test_results_depend_on_a_request_alone(hq, hkv, d, dtype, causal):
    """Bit for bit the same beside other requests, and whatever shared memory held before: rows of a tile that are not the request's decide nothing."""
    n = [300, 40, 129, 700, 1, 64]
    q, k, v = inputs(hq + d, n, n, hq, hkv, d, dtype, qscale=2.0)
    out, lse = ha.prompt_attention(q, k, v, offsets(n), causal=causal)
    big = torch.randn(2048, 2048, device="cuda").to(DT[dtype])
    for i in range(6):
        torch.mm(big * 10.0 ** (i - 2), big.T)                          # (leaves numbers of many sizes in shared memory)
        again = ha.prompt_attention(q, k, v, offsets(n), causal=causal)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    at = 0
    for a in n:
        alone = ha.prompt_attention(q[at:at + a], k[at:at + a], v[at:at + a], offsets([a]), causal=causal)
        assert torch.equal(out[at:at + a], alone[0]) and torch.equal(lse[at:at + a], alone[1]), a
        at += a


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (64, "fp16"), (128, "fp16")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_score_that_is_no_number_in_every_column(d, dtype, bad):
    """A request a column of a key tile, the first one walked and the second: every row that sees the key is NaN throughout, its log-sum-exp too; no other row changes."""
    nq, nk = [9] * 256, [260] * 256
    q, k, v = inputs(d, nq, nk, 1, 1, d, dtype)
    clean, lse_clean = ha.prompt_attention(q, k, v, offsets(nq), offsets(nk), out_dtype=torch.float32)
    k2 = k.view(256, 260, d).clone()
    k2[torch.arange(256), 4 + torch.arange(256)] = bad                  # (of an infinity and a query of both signs the score is NaN)
    out, lse = ha.prompt_attention(q, k2.view(-1, 1, d), v, offsets(nq), offsets(nk), out_dtype=torch.float32)
    sees = (torch.arange(9)[None] + 251 >= 4 + torch.arange(256)[:, None]).reshape(-1).cuda()       # row i sees keys 0 .. 251 + i
    assert out[sees].isnan().all() and lse[sees].isnan().all()
    assert torch.equal(out[~sees], clean[~sees]) and torch.equal(lse[~sees], lse_clean[~sees]) and int((~sees).sum()) == 36
