"""Exact attention over packed prompts against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
import serving_util as SU

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
ROUND = {"bf16": 2.0 ** -9, "fp16": 2.0 ** -12}         # what rounding to the type may be off, relative


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def offsets(lens):
    return ints(np.concatenate([[0], np.cumsum(lens)]))


def seen_by(nq, nk, causal):
    return np.maximum(nk - nq + 1 + np.arange(nq), 0) if causal else np.full(nq, nk)


def check(q, k, v, nq, nk, causal, out, lse, scale=None, weights=None):
    """out, lse (fp32) against 64 bits: weights rounded to the inputs' type in numerator and (at most) sum (2 roundings), scores that are fp32 sums of d
    products (2^-17 of sum |q k|), exp2 and sums a few 2^-22."""
    dtype = "bf16" if q.dtype == torch.bfloat16 else "fp16"
    G = q.shape[1] // k.shape[1]
    Q, K, V, out, lse = (SU.f64(x) for x in (q, k, v, out, lse))
    q0 = k0 = 0
    for a, b in zip(nq, nk):
        seen = seen_by(a, b, causal)
        for h in range(Q.shape[1]):
            o, l, mass, size = SU.attention(Q[q0:q0 + a, h], K[k0:k0 + b, h // G], V[k0:k0 + b, h // G], seen, scale)
            err = 2.0 ** -17 * size
            bound = (2 * ROUND[dtype] + 2 * err + 1e-5)[:, None] * mass + 1e-6
            assert np.all(np.abs(out[q0:q0 + a, h] - o) <= bound), (a, b, h, np.abs(out[q0:q0 + a, h] - o).max())
            there = seen > 0
            assert np.all(np.abs(lse[q0:q0 + a, h] - l)[there] <= (err + 2.0 ** -21 * np.abs(l) + 2e-6)[there]), (a, b, h)
            assert np.all(lse[q0:q0 + a, h][~there] == -np.inf) and not out[q0:q0 + a, h][~there].any()
        q0, k0 = q0 + a, k0 + b


def inputs(seed, nq, nk, hq, hkv, d, dtype, qscale=1.0):
    rng = np.random.default_rng(seed)
    q = torch.tensor(qscale * rng.standard_normal((sum(nq), hq, d))).to(DT[dtype]).cuda()
    k = torch.tensor(rng.standard_normal((sum(nk), hkv, d)) + rng.standard_normal((hkv, d))).to(DT[dtype]).cuda()
    v = torch.tensor(rng.standard_normal((sum(nk), hkv, d))).to(DT[dtype]).cuda()
    return q, k, v


SHAPES = [(2, 2, 64, "bf16"), (4, 1, 128, "bf16"), (6, 2, 64, "fp16"), (7, 1, 128, "fp16"), (16, 1, 128, "bf16"), (5, 1, 64, "bf16"), (1, 1, 128, "fp16")]


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
@pytest.mark.parametrize("causal", [True, False])
def test_lengths(hq, hkv, d, dtype, causal):
    n = [1, 2, 31, 0, 33, 127, 128, 129, 1, 300, 64, 257]
    q, k, v = inputs(hq * d, n, n, hq, hkv, d, dtype)
    out, lse = ha.prompt_attention(q, k, v, offsets(n), causal=causal, out_dtype=torch.float32)
    check(q, k, v, n, n, causal, out, lse)
    short, lse2 = ha.prompt_attention(q, k, v, offsets(n), causal=causal)
    assert torch.equal(short, out.to(DT[dtype])) and torch.equal(lse, lse2)


@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_more_and_fewer_keys_than_queries(hq, hkv, d, dtype):
    nq = [1, 1, 5, 130, 64, 3, 0, 200, 128, 40, 7]
    nk = [500, 1, 0, 131, 700, 2, 9, 60, 384, 40, 1]       # a continued prompt; no keys; queries that see none
    q, k, v = inputs(d + hq, nq, nk, hq, hkv, d, dtype)
    for causal in (True, False):
        out, lse = ha.prompt_attention(q, k, v, offsets(nq), offsets(nk), causal=causal, out_dtype=torch.float32)
        check(q, k, v, nq, nk, causal, out, lse)


@pytest.mark.parametrize("n,hq,hkv,d,dtype", [(1500, 2, 1, 128, "bf16"), (2049, 1, 1, 64, "fp16"), (1100, 3, 3, 64, "bf16"), (1000, 12, 1, 128, "fp16")])
def test_longer_prompts(n, hq, hkv, d, dtype):
    q, k, v = inputs(n, [n], [n], hq, hkv, d, dtype)
    out, lse = ha.prompt_attention(q, k, v, offsets([n]), out_dtype=torch.float32)
    check(q, k, v, [n], [n], True, out, lse)


def test_many_short_prompts():
    n = np.random.default_rng(5).integers(0, 40, 300).tolist()
    q, k, v = inputs(5, n, n, 4, 2, 64, "bf16")
    out, lse = ha.prompt_attention(q, k, v, offsets(n), out_dtype=torch.float32)
    check(q, k, v, n, n, True, out, lse)


def test_large_prompt_on_sampled_rows():
    """More key tiles and work items than SMs: rows of a long prompt against 64 bits on the GPU."""
    n, hq, hkv, d = 9000, 8, 2, 128
    gen = torch.Generator("cuda").manual_seed(1)
    q = torch.randn(n, hq, d, generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn(n, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    out, lse = ha.prompt_attention(q, k, v, offsets([n]), out_dtype=torch.float32)
    for i in [0, 1, 127, 128, 129, 4095, 4096, 6000, n - 2, n - 1]:
        for h in range(hq):
            o, l, mass, size = SU.attention(SU.f64(q[i, h])[None], SU.f64(k[:i + 1, h // 4]), SU.f64(v[:i + 1, h // 4]), [i + 1])
            err = 2.0 ** -17 * size[0]
            assert np.all(np.abs(SU.f64(out[i, h]) - o[0]) <= (2 * ROUND["bf16"] + 2 * err + 1e-5) * mass[0] + 1e-6)
            assert abs(float(lse[i, h]) - l[0]) <= err + 2.0 ** -21 * abs(l[0]) + 2e-6


def test_scores_of_every_size():
    """Scores that grow or shrink along the keys by hundreds, a scale of the caller's, scores that overflow to -infinity."""
    n, d = 700, 64
    for dtype in ("bf16", "fp16"):
        for up in (1, -1):
            q, k, v = inputs(3, [n], [n], 2, 1, d, dtype)
            ramp = torch.linspace(-1, 1, n, device="cuda")[:, None, None] * up
            k = (0.05 * k.float() + 20 * ramp).to(DT[dtype])
            q = q.abs()
            for scale in (0.0, 0.02, 1.5):
                out, lse = ha.prompt_attention(q, k, v, offsets([n]), scale=scale, out_dtype=torch.float32)
                check(q, k, v, [n], [n], True, out, lse, scale or None)
    # keys at minus infinity have no weight; a query that sees nothing else has none either
    q, k, v = inputs(4, [300], [300], 1, 1, d, "bf16")
    q = q.abs() + 0.1
    k[:7] = -float("inf")
    k[200] = -float("inf")
    out, lse = ha.prompt_attention(q, k, v, offsets([300]), out_dtype=torch.float32)
    assert not out[:7].any() and torch.isinf(lse[:7]).all() and torch.isfinite(out[7:]).all()
    keep = [j for j in range(300) if j >= 7 and j != 200]
    o, l, mass, _ = SU.attention(SU.f64(q[299]), SU.f64(k[keep, 0]), SU.f64(v[keep, 0]), [len(keep)])
    assert np.all(np.abs(SU.f64(out[299]) - o) <= 2.0 ** -8 * mass + 1e-5) and abs(float(lse[299]) - l[0]) < 1e-4


@pytest.mark.parametrize("d,G", [(64, 1), (128, 4)])
def test_what_a_query_does_not_see_has_no_influence(d, G):
    """Infinities and NaN in later keys and values, in other requests and beyond the last row."""
    n = [100, 60, 200]
    q, k, v = inputs(6, n, n, 2 * G, 2, d, "bf16")
    clean, lse_clean = ha.prompt_attention(q, k, v, offsets(n), out_dtype=torch.float32)
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        k2[250:], v2[250:] = bad, bad                       # request 2 from its query 90 on
        v2[120, 1, 3] = bad                                 # request 1, a value that its queries from 20 on see
        k2[60, 0] = bad                                     # request 0, a key that its queries from 60 on see
        out, lse = ha.prompt_attention(q, k2, v2, offsets(n), out_dtype=torch.float32)
        fine = torch.ones_like(out, dtype=torch.bool)
        fine[250:] = False
        fine[120:160, G:, 3] = False
        fine[60:100, :G] = False
        # (a row that is computed in another way, for the sake of the others in its tile, may differ in the last places)
        assert torch.isfinite(out[fine]).all() and (out - clean)[fine].abs().max() <= 2.0 ** -7 * clean.abs().max()
        rows = torch.ones_like(lse, dtype=torch.bool)
        rows[250:], rows[60:100, :G] = False, False
        assert (lse - lse_clean)[rows].abs().max() <= 1e-4
        assert not torch.isfinite(out[120:160, G:, 3]).any() and not torch.isfinite(out[250:]).any()
        if bad == bad and bad < 0:
            continue
        assert not torch.isfinite(out[60:100, :G]).any()


def test_no_keys_at_all():
    q, k, v = inputs(8, [5, 130], [0, 0], 4, 2, 128, "bf16")
    out, lse = ha.prompt_attention(q, k, v, offsets([5, 130]), offsets([0, 0]))
    assert not out.any() and torch.isinf(lse).all() and (lse < 0).all()
    out, lse = ha.prompt_attention(q[:0], k, v, offsets([0, 0]), offsets([0, 0]))
    assert out.shape == (0, 4, 128) and lse.shape == (0, 4)


def test_offsets_that_do_not_fit_the_tensors():
    """Offsets beyond the rows that there are, or that go back, read and write nothing outside."""
    q, k, v = inputs(9, [40], [40], 2, 2, 64, "bf16")
    guard = [x.clone() for x in (q, k, v)]
    for cu_q, cu_k in (([0, 90], [0, 40]), ([0, 40], [0, 500]), ([-7, 40], [-9, 40]), ([0, 30, 10, 40], [0, 20, 5, 40])):
        out, lse = ha.prompt_attention(q, k, v, ints(cu_q), ints(cu_k))
        assert out.shape == q.shape
    assert all(torch.equal(a, b) for a, b in zip(guard, (q, k, v)))
    assert ha.last_device_status() == 0


def test_rows_beyond_the_last_request_are_not_written():
    q, k, v = inputs(7, [70], [70], 2, 1, 64, "bf16")
    v[50:] = float("nan")
    k[50:] = float("inf")
    want = ha.prompt_attention(q[:50], k[:50], v[:50], offsets([20, 30]))
    got = ha.prompt_attention(q, k, v, offsets([20, 30]))
    assert torch.equal(got[0][:50], want[0]) and torch.equal(got[1][:50], want[1])


def test_views_streams_and_a_graph():
    n = [90, 1, 140]
    T = sum(n)
    qkv = torch.randn(T, 8, 128, device="cuda").bfloat16()
    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    want = ha.prompt_attention(q.contiguous(), k.contiguous(), v.contiguous(), offsets(n))
    for a, b, c in ((q, k, v), tuple(x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)),
                    (torch.cat([q, q], -1)[..., 128:], torch.cat([k, k], -1)[..., :128], v)):
        got = ha.prompt_attention(a, b, c, offsets(n))
        assert all(torch.equal(x, y) for x, y in zip(want, got))
    one = torch.randn(1, 2, 128, device="cuda").bfloat16().expand(T, 2, 128)          # every key the same row: a stride of zero
    got, want0 = ha.prompt_attention(q, one, v, offsets(n)), ha.prompt_attention(q, one.contiguous(), v, offsets(n))
    assert torch.equal(got[0], want0[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ha.prompt_attention(q, k, v, offsets(n))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    cu = offsets(n)
    side.wait_stream(torch.cuda.current_stream())
    got = ha.prompt_attention(q, k, v, cu, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    ha.prompt_attention(q, k, v, cu)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = ha.prompt_attention(q, k, v, cu)
    for lens in ([90, 1, 140], [20, 200, 11]):
        cu.copy_(offsets(lens))
        graph.replay()
        want = ha.prompt_attention(q, k, v, cu)
        assert all(torch.equal(x, y) for x, y in zip(held, want))
