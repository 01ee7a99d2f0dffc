"""Steps of a server most of whose places are without a request, or whose requests are mostly without new tokens."""
import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU
import test_gpu_cache_chunk as TC

pytestmark = pytest.mark.gpu

# places, new tokens of those that have any, tokens of others
STEPS = {
    "one part": (64, {0: 300}, 0),
    "one part, last": (64, {63: 300}, 0),
    "far apart": (500, {3: 40, 97: 700, 98: 1, 499: 1300}, 0),
    "beside contexts that wait": (100, {1: 2, 50: 650, 99: 5}, 130),
    "many places": (4096, {0: 1, 2047: 260, 4000: 33, 4095: 4100}, 0),
    "many places, few rows": (4096, {31: 1, 32: 64, 4095: 3}, 0),
}


@pytest.mark.parametrize("heads", [(2, 2, 64), (4, 1, 128)])
@pytest.mark.parametrize("step", STEPS)
def test_steps_of_few_requests(step, heads):
    places, new, waiting = STEPS[step]
    counts = [new.get(r, 0) for r in range(places)]
    lens = [n + 200 * (r % 3) if n else waiting for r, n in enumerate(counts)]
    q, cache, table, k, v, (out, lse), _ = TC.both(lens, counts, heads, 16, torch.bfloat16)
    before = torch.rand(places, heads[1], table.shape[1] * 16, device="cuda")
    TC.check_weights(q, cache, table, k, lens, counts, lse, before=before, decay=0.5)


@pytest.mark.parametrize("heads", [(2, 2, 64), (4, 1, 128), (32, 1, 64)])
@pytest.mark.parametrize("counts", [[1] * 90, [4] * 40 + [1] * 60, [300] + [0] * 63, [700, 2, 0, 900] + [1] * 20])
def test_the_most_new_tokens_change_nothing_but_the_way(counts, heads):
    """Right, too small, too large: results within the same bounds, and in the workspace that a call without it has."""
    lens = [n + 37 * (r % 9) for r, n in enumerate(counts)]
    dtype = torch.float16 if heads[2] == 64 else torch.bfloat16
    q, cache, table, k, v, (out, lse), want = TC.both(lens, counts, heads, 16, dtype, width=64)
    lengths, cu = CU.ints(lens), CU.offsets(counts)
    exact, bound = CU.weights(q.double(), k, lens, counts, lse, cap=table.shape[1] * 16)
    for most in (1, max(counts), 100000):
        got = ha.cache_chunk_attention(q, cache, table, lengths, cu, most_new=most)
        CU.check_attention(got, want, dtype, max(lens), sum(counts))
        w = ha.cache_weights(q, cache, table, lengths, lse, cu, most_new=most)
        assert bool(((w.double() - exact).abs() <= bound).all())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    there = ha.cache_chunk_attention(q, cache, table, lengths, cu, stream=side.cuda_stream, most_new=100000)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(there[0], got[0]) and torch.equal(there[1], got[1])
