"""Chunks, weights, pages and eviction together: the example's server with contexts that are cut, against the same decoder with plain attention over what its
caches hold."""
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
KEEP, RECENT, FIRST = 40, 8, 2


def example():
    spec = importlib.util.spec_from_file_location("serve_example", os.path.join(ROOT, "examples", "serve.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_step(model, contexts, request, tokens, seen):
    """Logits of a request's new tokens.  contexts[layer][request]: K, V [tokens, heads, d] and weights [tokens, heads] of the tokens that are left; seen: tokens that there have been."""
    G = model.q_heads // model.kv_heads
    positions = torch.arange(seen, seen + len(tokens), device="cuda")

    def attend(layer, q, k, v):
        old_k, old_v, old_w = contexts[layer][request]
        held = [torch.tensor(SU.held(x.float().cpu().numpy()), device="cuda") for x in (k, v)]
        K, V = torch.cat([old_k, held[0]]), torch.cat([old_v, held[1]])
        z = torch.einsum("qhd,khd->hqk", q.double(), K.double().repeat_interleave(G, 1)) / math.sqrt(model.d)
        visible = torch.arange(K.shape[0], device="cuda")[None] <= old_k.shape[0] + torch.arange(len(tokens), device="cuda")[:, None]
        p = z.masked_fill(~visible, -math.inf).softmax(-1)
        w = p.sum(1).view(-1, G, K.shape[0]).sum(1).T.contiguous()
        w[:old_w.shape[0]] += old_w
        contexts[layer][request] = K, V, w
        return torch.einsum("hqk,khd->qhd", p, V.double().repeat_interleave(G, 1)).to(q.dtype)

    return model.run(torch.tensor(tokens, device="cuda"), positions, attend)[-1]


def test_server_with_contexts_that_are_cut():
    E = example()
    model = E.Decoder(layers=2, q_heads=6, kv_heads=2, d=64)
    server = E.Server(model, requests=3, pages=24, page_tokens=16, longest=128, keep=KEEP, recent=RECENT, first=FIRST)
    none = (torch.zeros(0, 2, 64, device="cuda"), torch.zeros(0, 2, 64, device="cuda"), torch.zeros(0, 2, device="cuda", dtype=torch.float64))
    contexts = [{r: none for r in range(3)} for _ in model.layers]
    seen, cuts = [0, 0, 0], 0
    rng = np.random.default_rng(0)

    def words(n):
        return rng.integers(0, 512, n).tolist()

    # prompts at once and in parts, tokens side by side, some at a time, a request that ends and another in its place, one that does not fit
    steps = [[words(20), words(1), None], [words(1), words(33), words(60)], [words(30), words(3), words(1)], [words(1), words(20), words(45)], [False, words(1), words(2)],
             [words(128), words(1), words(1)], [words(100), words(50), words(1)], [words(1), words(2), False], [words(5), words(1), words(100)], [words(1), words(1), words(1)]]
    for new in steps:
        got = server.step(new)
        for r, tokens in enumerate(new):
            if tokens is False:
                seen[r] = 0
                for c in contexts:
                    c[r] = none
        for r, logits in got.items():
            want = plain_step(model, contexts, r, new[r], seen[r])
            seen[r] += len(new[r])
            # bf16 activations through two layers; attention's own errors (2^-11 of values and weights) go through them once
            assert (logits - want).norm() <= 2e-2 * want.norm(), (r, float((logits - want).norm() / want.norm()))
        lengths = [contexts[0][r][0].shape[0] for r in range(3)]
        assert server.lengths.tolist() == lengths
        for layer, c in enumerate(contexts):
            for r, n in enumerate(lengths):
                w = server.weights[layer][r, :, :n].T.double()
                # activations as above: probabilities are as far off (scores of some units, each 2^-8 and its like)
                assert (w - c[r][2]).norm() <= 2e-2 * c[r][2].norm()
        kept = server.cut()
        after = server.lengths.tolist()
        for r, (n, m) in enumerate(zip(lengths, after)):
            assert m == min(n, KEEP)
            if m < n:
                cuts += 1
                for layer, c in enumerate(contexts):
                    for h in range(2):
                        stay = kept[layer][r, h, :m].tolist()
                        assert set(range(FIRST)) <= set(stay) and set(range(n - RECENT, n)) <= set(stay) and stay == sorted(set(stay))
                    at = kept[layer][r, :, :m].T.long()
                    K, V, w = c[r]
                    c[r] = (*(x.gather(0, at[..., None].expand(-1, -1, 64)) for x in (K, V)), w.gather(0, at))
        assert int(server.n_free) == 24 - sum(-(-n // 16) for n in after)
        pages = [p for p in server.table.flatten().tolist() + server.free.tolist() if p >= 0]
        assert sorted(pages) == list(range(24))
    assert cuts >= 6


def test_example_runs(capsys):
    example().main(keep=256)
    assert "pages free" in capsys.readouterr().out
