"""Exact attention over packed prompts where numbers come near the ends of their types: scores far apart."""
import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha
from test_gpu_prompt import DT, check, offsets

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
