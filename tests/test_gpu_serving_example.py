"""The serving operators together: the example's server against the same decoder with plain attention over what its caches hold."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2310_05869_b200 as ha  # noqa: F401  (the example imports it)
import serving_util as SU

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("serve_example", os.path.join(ROOT, "examples", "serve.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_step(model, contexts, request, tokens):
    """Logits of a request's new tokens; contexts[layer][request]: (K, V) of its earlier tokens as the cache holds them."""
    G = model.q_heads // model.kv_heads
    past = contexts[0][request][0].shape[0]
    positions = torch.arange(past, past + len(tokens), device="cuda")

    def attend(layer, q, k, v):
        old_k, old_v = contexts[layer][request]
        held = [torch.tensor(SU.held(x.float().cpu().numpy()), device="cuda") for x in (k, v)]
        # a token alone sees its own key and value from the cache; a prompt its own before they are rounded
        mine = held if len(tokens) == 1 else (k.float(), v.float())
        keys, values = (torch.cat([a, b]).repeat_interleave(G, 1) for a, b in ((old_k, mine[0]), (old_v, mine[1])))
        z = torch.einsum("qhd,khd->hqk", q.float(), keys) / math.sqrt(model.d)
        seen = torch.arange(keys.shape[0], device="cuda")[None] <= positions[:, None]
        out = torch.einsum("hqk,khd->qhd", z.masked_fill(~seen, -math.inf).softmax(-1), values)
        contexts[layer][request] = torch.cat([old_k, held[0]]), torch.cat([old_v, held[1]])
        return out.to(q.dtype)

    return model.run(torch.tensor(tokens, device="cuda"), positions, attend)[-1]


def test_server_against_plain_attention():
    E = example()
    model = E.Decoder(layers=2, q_heads=6, kv_heads=2, d=64)
    server = E.Server(model, requests=3, pages=12, page_tokens=16, longest=96)
    none = (torch.zeros(0, 2, 64, device="cuda"), torch.zeros(0, 2, 64, device="cuda"))
    contexts = [{r: none for r in range(3)} for _ in model.layers]
    rng = np.random.default_rng(0)

    def words(n):
        return rng.integers(0, 512, n).tolist()

    # prompts and tokens side by side, prompts in parts, a request that ends and another in its place, one that finds no pages
    steps = [[words(20), words(1), None], [words(1), words(33), words(40)], [words(1), words(1), words(9)], [False, words(1), words(1)],
             [words(90), words(1), words(1)], [words(3), words(1), words(1)], [words(50), False, False], [words(1), words(17), words(30)]]
    free = 12
    for new in steps:
        got = server.step(new)
        for r, tokens in enumerate(new):
            if tokens is False:
                for c in contexts:
                    c[r] = none
        for r, logits in got.items():
            want = plain_step(model, contexts, r, new[r])
            # bf16 activations through two layers; attention's own errors (2^-9 of values and weights) go through them once
            assert (logits - want).norm() <= 2e-2 * want.norm(), (r, float((logits - want).norm() / want.norm()))
        lengths = [contexts[0][r][0].shape[0] for r in range(3)]
        assert server.lengths.tolist() == lengths
        free = 12 - sum(-(-n // 16) for n in lengths)
        assert int(server.n_free) == free
    assert free >= 0


def test_example_runs(capsys):
    example().main()
    assert "pages free" in capsys.readouterr().out
