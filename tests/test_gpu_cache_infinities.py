"""Caches that were filled by other means than cache_store, which holds what is not finite as NaN: an infinite scale or minimum among the keys is the matter of the rows that see
its token, and of that token's weight."""
import math

import pytest
import torch

import paper_2310_05869_b200 as ha
import chunk_util as CU
import test_gpu_cache_chunk as TC

pytestmark = pytest.mark.gpu

LENGTH, PAGE = 640, 64


def place_of(cache, table, token, d, group, minimum):
    """The fp16 scale (or minimum) of a token's key of head 0 in its block, a view of one element."""
    block = cache[int(table[0, token // PAGE]), 0, token % PAGE // 16].view(torch.float16)
    t = token % 16
    at = 8 * d + (t // 2 * (d // 32) + group) * 4 + t % 2 + (2 if minimum else 0)
    return block[at:at + 1]


@pytest.mark.parametrize("number", [math.inf, -math.inf])
@pytest.mark.parametrize("minimum", [False, True])
@pytest.mark.parametrize("rows", [20, 100, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_keys_beside_large_ones(d, rows, minimum, number):
    """Token t has keys some twenty times as large as the others, by its scales (from 0 on) or by its minima (around 40); token t + 8 of the same block, whose numbers a lane holds beside t's, an
    infinity.  Rows that do not see t + 8 get the bits that they get without it."""
    if number < 0 and not minimum:
        number = math.nan                                          # (scales are not negative)
    t = LENGTH - rows + min(rows // 2, 3)
    t = t // 16 * 16 + 3 if rows > 40 else t // 16 * 16 + 1        # (t + 8 is in the same block)
    if t + 8 < LENGTH - rows + 1:
        t += 16
    assert t + 8 < LENGTH

    def put(k, v):
        k[t] = (40 + k[t].float() * 0.1 if minimum else k[t].float().abs().clamp(min=0.1) * 20).to(k.dtype)

    cache, table, k, v = CU.filled([LENGTH], 1, d, PAGE, torch.bfloat16, put=put)
    q = TC.queries(rows, 1, d, torch.bfloat16, scale=0.05)
    lengths, cu = CU.ints([LENGTH]), CU.offsets([rows])
    want = ha.cache_chunk_attention(q, cache, table, lengths, cu, out_dtype=torch.float32)
    w = ha.cache_weights(q, cache, table, lengths, want[1], cu)
    for group in range(d // 32):
        place = place_of(cache, table, t + 8, d, group, minimum)
        before = place.clone()
        place.fill_(number)
        out, lse = ha.cache_chunk_attention(q, cache, table, lengths, cu, out_dtype=torch.float32)
        got = ha.cache_weights(q, cache, table, lengths, want[1], cu)
        place.copy_(before)
        unseen = t + 8 - (LENGTH - rows)                           # rows before this one do not see token t + 8
        assert torch.equal(out[:unseen], want[0][:unseen]) and torch.equal(lse[:unseen], want[1][:unseen])
        others = torch.arange(w.shape[2], device="cuda") != t + 8
        assert torch.equal(got[..., others], w[..., others])
