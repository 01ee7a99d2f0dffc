"""Exact attention over packed prompts where numbers come near the ends of their types: scores far apart, values that nobody may see, rows beside others."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
from test_gpu_prompt import DT, check, inputs, offsets

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
