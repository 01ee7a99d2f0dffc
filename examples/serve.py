"""A small server of a decoder: prompts of different lengths come and go, their keys and values are kept in a paged 4-bit cache.

    python examples/serve.py                 # random weights; prints what it generated and how long a step took
    python examples/serve.py --keep 512      # the same prompts with contexts that are cut to 512 tokens; no layer is approximated then

Every step schedules the cache's pages (cache_plan), runs the new tokens of all requests as one packed batch - whole prompts for
requests that have just come, one token for the others - and, layer by layer, stores their keys and values (cache_store) and attends:
prompts to themselves (prompt_attention), or, from `long_prompt` tokens on, with HyperAttention in the layers that are to be
approximated; single tokens to everything that is cached of their request (cache_attention).  A prompt that comes in parts attends
to its cached part, read back (cache_read), and to itself.

With `keep`, no request has more than that many tokens for long: all rows of a step attend to what is cached of their requests, their
own tokens included (cache_chunk_attention), the weight that every cached token gets is added up (cache_weights), and requests that
have grown too long are cut to the first and the last tokens and those of most weight (cache_evict_plan, and cache_evict for every
layer).  The weights are those of exact attention, so a model with approximated layers is refused.  This is a loop to read, not a
server: everything outside the library's calls is plain torch."""
from __future__ import annotations

import math
import os
import sys
import time

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_05869_b200 as ha


class Decoder:
    """Weights of a decoder with grouped heads and rotary positions (random ones: there is nothing to download)."""

    def __init__(self, layers=2, q_heads=8, kv_heads=2, d=64, vocabulary=512, approximated=(), dtype=torch.bfloat16, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        width = q_heads * d

        def weight(*shape):
            return (torch.randn(*shape, generator=gen, device="cuda") / math.sqrt(shape[0])).to(dtype)

        self.q_heads, self.kv_heads, self.d, self.dtype, self.approximated = q_heads, kv_heads, d, dtype, set(approximated)
        self.embedding = weight(vocabulary, width) * math.sqrt(vocabulary)
        self.layers = [{"qkv": weight(width, (q_heads + 2 * kv_heads) * d), "out": weight(width, width), "up": weight(width, 2 * width), "down": weight(2 * width, width)}
                       for _ in range(layers)]

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def turned(self, x, positions):
        """x [rows, heads, d] with its pairs (i, i + d / 2) turned by the rows' positions."""
        half = self.d // 2
        angle = positions[:, None, None] * 10000.0 ** (-torch.arange(half, device=x.device) / half)
        a, b = x.float()[..., :half], x.float()[..., half:]
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1).to(x.dtype)

    def run(self, tokens, positions, attend):
        """Logits of a packed batch; attend(layer, q, k, v) -> [rows, q_heads, d]."""
        x = self.embedding[tokens]
        H, G, d = self.q_heads, self.kv_heads, self.d
        for i, w in enumerate(self.layers):
            q, k, v = (self.norm(x) @ w["qkv"]).view(-1, H + 2 * G, d).split((H, G, G), 1)     # (views: rows and heads of a wider tensor)
            x = x + attend(i, self.turned(q, positions), self.turned(k, positions), v).reshape(x.shape) @ w["out"]
            x = x + torch.nn.functional.silu(self.norm(x) @ w["up"]) @ w["down"]
        return (self.norm(x) @ self.embedding.T).float()


class Server:
    def __init__(self, model, requests=8, pages=64, page_tokens=64, longest=2048, long_prompt=1 << 30, keep=0, recent=32, first=4):
        if keep and model.approximated:
            raise ValueError("keep needs a model without approximated layers")
        self.model, self.page, self.long_prompt, self.keep, self.recent, self.first = model, page_tokens, long_prompt, keep, recent, first
        self.caches = [ha.cache_pages(pages, model.kv_heads, model.d, page_tokens) for _ in model.layers]

        def ints(*shape, fill=0):
            return torch.full(shape, fill, dtype=torch.int32, device="cuda")

        self.lengths, self.table = ints(requests), ints(requests, -(-longest // page_tokens), fill=-1)
        self.free, self.n_free = torch.arange(pages, dtype=torch.int32, device="cuda"), ints(1, fill=pages)
        if keep:                                                   # what every cached token has got, and how many tokens of a request are gone
            self.weights = [torch.zeros(requests, model.kv_heads, self.table.shape[1] * page_tokens, device="cuda") for _ in model.layers]
            self.gone, self.most = ints(requests), ints(requests, fill=keep)

    def step(self, new):
        """new: for every request None (nothing), False (it has ended) or its new tokens (a list); returns the logits of every request's last
        new token {request: [vocabulary]} of those that were admitted."""
        model = self.model
        count = [-1 if t is False else len(t or ()) for t in new]
        rows = sum(max(n, 0) for n in count)
        before = self.lengths
        plan = ha.cache_plan(before, torch.tensor(count, dtype=torch.int32, device="cuda"), self.table, self.free, self.n_free, self.page, rows)
        self.lengths, self.table, self.free, self.n_free = plan.lengths, plan.table, plan.free, plan.n_free
        if self.keep:
            self.gone.masked_fill_(plan.lengths == 0, 0)
        if rows == 0:
            return {}
        tokens = torch.tensor([t for request in new if request for t in request], device="cuda")
        admitted = {r for r, ok in enumerate((plan.lengths > before).tolist()) if ok}
        first = plan.cu_new.tolist()
        if self.keep:
            # rows of the requests that were admitted, one after the other (all of them, nearly always)
            mine = sorted(admitted)
            if not mine:
                return {}
            pick = torch.cat([torch.arange(first[r], first[r + 1]) for r in mine]).cuda()
            cu = torch.tensor([0] + [count[r] if r in admitted else 0 for r in range(len(new))]).cumsum(0).int().cuda()
            moved = torch.repeat_interleave(self.gone, plan.cu_new.diff(), output_size=rows)
            most = max(count)

            def attend_cached(layer, q, k, v):
                cache = self.caches[layer]
                ha.cache_store(cache, k, v, plan.slots)
                q1 = q if pick.shape[0] == rows else q[pick]
                got, lse = ha.cache_chunk_attention(q1, cache, plan.table, plan.lengths, cu, most_new=most)
                ha.cache_weights(q1, cache, plan.table, plan.lengths, lse, cu, weights=self.weights[layer], out=self.weights[layer], most_new=most)
                return got if pick.shape[0] == rows else torch.zeros_like(q).index_copy_(0, pick, got)

            logits = model.run(tokens, plan.positions.clamp(min=0) + moved, attend_cached)
            return {r: logits[first[r + 1] - 1] for r in mine}

        held = before.tolist()                                     # (a real server knows the lengths it has sent)
        single = [r for r, n in enumerate(count) if n == 1 and r in admitted]
        prompts = [r for r, n in enumerate(count) if n > 1 and r in admitted]
        rows_of_single = torch.tensor([first[r] for r in single], device="cuda", dtype=torch.long)
        at = torch.tensor(single, device="cuda", dtype=torch.long)
        table1, lengths1 = plan.table[at].contiguous(), plan.lengths[at].contiguous()

        def attend(layer, q, k, v):
            out = torch.zeros_like(q)
            cache = self.caches[layer]
            ha.cache_store(cache, k, v, plan.slots)
            if single:
                out[rows_of_single] = ha.cache_attention(q[rows_of_single], cache, table1, lengths1)[0]
            whole = []
            for r in prompts:
                a, b = first[r], first[r + 1]
                if held[r] == 0 and b - a >= self.long_prompt and layer in model.approximated:
                    wide = [x[a:b].transpose(0, 1).repeat_interleave(model.q_heads // x.shape[1], 0)[None].contiguous() for x in (q, k, v)]
                    out[a:b] = ha.forward(*wide, 256, 256, 7, causal=True, n0=1024)[0][0].transpose(0, 1)
                else:
                    whole.append(r)
            if whole:                                              # one call for all of them, cached parts in front
                cu_q = torch.tensor([0] + [first[r + 1] - first[r] for r in whole], device="cuda").cumsum(0).int()
                past = torch.tensor([0] + [held[r] for r in whole], device="cuda").cumsum(0).int()
                mine = torch.cat([torch.arange(first[r], first[r + 1], device="cuda") for r in whole])
                old_k, old_v = ha.cache_read(cache, plan.table[whole].contiguous(), past, sum(held[r] for r in whole), dtype=k.dtype)
                parts = [(old[past[i]:past[i + 1]], x[first[r]:first[r + 1]]) for old, x in ((old_k, k), (old_v, v)) for i, r in enumerate(whole)]
                n = len(whole)
                keys, values = (torch.cat([x for pair in parts[j * n:(j + 1) * n] for x in pair]) for j in range(2))
                out[mine] = ha.prompt_attention(q[mine], keys, values, cu_q, (cu_q + past).int())[0]
            return out

        logits = model.run(tokens, plan.positions.clamp(min=0), attend)
        return {r: logits[first[r + 1] - 1] for r in single + prompts}

    def cut(self):
        """Requests of more than `keep` tokens are cut to that; returns the tokens (before) that stay, a tensor for every layer."""
        plan = ha.cache_evict_plan(self.lengths, self.most, self.table, self.free, self.n_free, self.page)
        kept = []
        for layer, cache in enumerate(self.caches):
            self.weights[layer], stay = ha.cache_evict(cache, self.weights[layer], self.table, self.lengths, plan.table, plan.lengths, recent=self.recent, first=self.first)
            kept.append(stay)
        self.gone += self.lengths - plan.lengths
        self.lengths, self.table, self.free, self.n_free = plan
        return kept


def main(keep=0):
    server = Server(Decoder(layers=4, approximated=() if keep else {3}), requests=4, pages=200, longest=8192, long_prompt=4096, keep=keep)
    gen = torch.Generator().manual_seed(1)
    waiting = [torch.randint(0, 512, (n,), generator=gen).tolist() for n in (5, 700, 5000, 64, 1, 300)]
    said = {r: [] for r in range(len(waiting))}
    running, new, todo = [None] * 4, [None] * 4, list(enumerate(waiting))
    steps, began = 0, time.perf_counter()
    while todo or any(r is not None for r in running):
        for s in range(4):                                         # an empty place takes the next prompt
            if running[s] is None and new[s] is None and todo:
                running[s], new[s] = todo.pop(0)
        got = server.step(new)
        if keep:
            server.cut()
        new = [None] * 4
        for s, logits in got.items():
            said[running[s]].append(int(logits.argmax()))
            if len(said[running[s]]) == 12:
                running[s], new[s] = None, False                   # ended: its pages go back with the next step
            else:
                new[s] = said[running[s]][-1:]
        steps += 1
    torch.cuda.synchronize()
    for r, tokens in said.items():
        print(f"prompt of {len(waiting[r])}: {tokens}")
    print(f"{steps} steps, {(time.perf_counter() - began) / steps * 1e3:.2f} ms each; {int(server.n_free)} of {server.free.shape[0]} pages free")


if __name__ == "__main__":
    main(int(sys.argv[sys.argv.index("--keep") + 1]) if "--keep" in sys.argv else 0)
