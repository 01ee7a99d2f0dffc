"""Performance cases of the operators that serve a long-context model next to the library's prompt attention.

Five operators, two or three cases each:

  plan    one scheduling step of a paged cache: pages handed out and taken back, block tables, slots and positions of the
          step's tokens, from the requests' lengths, on the GPU
  store   K and V of new tokens into a paged cache that holds them in 4 bits (read back, as the values they stand for)
  read    cached K and V as ordinary tensors (a later part of a long prompt attends to them)
  attend  attention of one new token a request over the 4-bit cache
  prompt  exact causal attention over packed prompts of different lengths, grouped heads

Head counts and widths: 32 heads of 64 or 128 as in the benchmark configurations, with as many key / value heads, a quarter of
them, or two.  The cache's pages have 64 tokens unless a case says otherwise.

Layout of the cache, [pages, kv_heads, page / 16, 20 d] bytes: blocks of 16 tokens of one head, in each 8 d bytes of K codes, 8 d of V
codes, then scales and minima of the groups of 32 coordinates (fp16), 2 d bytes for K, 2 d for V.  A value is minimum + scale * code.

Inputs are synthetic, made on the GPU: queries and values N(0, 1), keys N(0, 1) around an offset per channel (as keys have)."""
import math
import random

import numpy as np
import torch

own = False

GROUP = 32


def _case(op, **kw):
    return dict(op=op, **kw)


def listed():
    named = {
        # A decode step of a server: every request gets one token, a few end, a few prompts come in.
        "plan_decode_256": _case("plan", requests=256, longest=8192, page=64, prompt=300),
        # The most that is scheduled in one step: 1024 requests of up to 131072 tokens, long prompts among them.
        "plan_prompts_1024": _case("plan", requests=1024, longest=131072, page=64, prompt=2000),
        # One token a request goes into the cache of a layer with a quarter of the heads for keys: latency.
        "store_decode_64": _case("store", requests=64, new=64, past=3000, kv_heads=8, d=128, page=64, dtype="bf16"),
        # Packed prompts of a layer of 32 heads of 64, none of them a multiple of anything.
        "store_prompts_32k": _case("store", requests=7, new=32768, past=0, kv_heads=32, d=64, page=64, dtype="fp16"),
        # A shared prefix of a few hundred tokens, small pages.
        "read_prefix_500": _case("read", requests=1, tokens=500, kv_heads=2, d=128, page=16, dtype="bf16"),
        # The cached part of long prompts, before their next part attends to it.
        "read_contexts_64k": _case("read", requests=5, tokens=65536, kv_heads=8, d=128, page=64, dtype="bf16"),
        # A handful of short chats: latency of one decode step.
        "attend_chats_4": _case("attend", requests=4, longest=600, q_heads=32, kv_heads=2, d=128, page=64, dtype="bf16"),
        # A batch of ordinary contexts, ragged lengths, one request without any token.
        "attend_batch_64": _case("attend", requests=64, longest=8192, q_heads=32, kv_heads=8, d=128, page=64, dtype="bf16"),
        # The headline context, 131072 tokens, as many key heads as query heads, two requests.
        "attend_131k": _case("attend", requests=2, longest=131072, q_heads=32, kv_heads=32, d=64, page=64, dtype="fp16"),
        # Short prompts packed together, lengths from one token on.
        "prompt_short_1k": _case("prompt", requests=13, tokens=1021, past=0, q_heads=32, kv_heads=8, d=128, dtype="bf16"),
        # The second part of prompts whose first part is cached: more keys than queries.
        "prompt_chunk_6k": _case("prompt", requests=3, tokens=6001, past=2500, q_heads=32, kv_heads=32, d=64, dtype="fp16"),
        # A full layer's share of one long prompt.
        "prompt_16k": _case("prompt", requests=1, tokens=16384, past=0, q_heads=16, kv_heads=2, d=128, dtype="bf16"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def draw(rng):
    def span(lo, hi):              # log-uniform, both ends included
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    def heads():
        return rng.choice([(32, 32, 64), (32, 8, 128), (32, 2, 128), (16, 2, 128), (32, 8, 64), (12, 12, 64), (28, 4, 128), (9, 3, 64)])

    op = rng.choice(["plan", "store", "read", "attend", "attend", "prompt", "prompt"])
    hq, hkv, d = heads()
    page, dtype = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "fp16"])
    if op == "plan":
        return _case("plan", requests=span(1, 1024), longest=span(512, 131072), page=page, prompt=span(16, 2000))
    if op == "store":
        new = min(span(1, 32768), 32768 * 32 * 64 // (hkv * d))
        return _case("store", requests=min(new, span(1, 256)), new=new, past=rng.choice([0, span(1, 4000)]), kv_heads=hkv, d=d, page=page, dtype=dtype)
    if op == "read":
        tokens = min(span(100, 65536), 65536 * 8 * 128 // (hkv * d))
        return _case("read", requests=min(tokens, span(1, 64)), tokens=tokens, kv_heads=hkv, d=d, page=page, dtype=dtype)
    if op == "attend":
        longest = span(100, 131072)
        most = 2 * 131072 * 32 * 64 // (hkv * d)                  # K entries of the largest listed case
        return _case("attend", requests=max(1, min(span(1, 256), most // longest)), longest=longest, q_heads=hq, kv_heads=hkv, d=d, page=page, dtype=dtype)
    tokens = span(100, 8192)
    return _case("prompt", requests=min(tokens, span(1, 32)), tokens=tokens, past=rng.choice([0, 0, span(1, 4000)]), q_heads=hq, kv_heads=hkv, d=d, dtype=dtype)


def _dtype(case):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[case["dtype"]]


# ---- lengths: made from the case alone, so that the work of a pass can be told without its inputs -----------------------
def _parts(total, parts, rng):
    """`total` tokens over `parts` requests, one at least each."""
    weights = [rng.random() ** 2 + 0.02 for _ in range(parts)]
    scale = (total - parts) / sum(weights)
    got = [1 + int(w * scale) for w in weights]
    got[-1] += total - sum(got)
    return got


def _lengths(case):
    """(tokens that are cached before, new tokens) of every request."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    R = case["requests"]
    if case["op"] == "store":
        return [rng.randint(0, 2 * case["past"]) for _ in range(R)], _parts(case["new"], R, rng)
    if case["op"] == "read":
        return _parts(case["tokens"], R, rng), [0] * R
    if case["op"] == "attend":
        lens = [rng.randint(1, case["longest"]) for _ in range(R)]
        lens[0] = case["longest"]
        if R > 8:
            lens[1], lens[2] = 0, 1
        return lens, [0] * R
    new = _parts(case["tokens"], R, rng)
    return [rng.randint(0, 2 * case["past"]) for _ in range(R)], new


def _offsets(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


# ---- the cache's layout ------------------------------------------------------------------------------------------------
def _places(d):
    """Where a block of 16 tokens holds coordinate x of token t: byte and bit of K's and V's codes, bytes of the scales' first halves."""
    t, x = torch.meshgrid(torch.arange(16), torch.arange(d), indexing="ij")
    lane, half = (t % 8) * 4 + (x // 8) % 4, t // 8
    e, w = x % 8, x // 32
    nib = (e % 2) * 4 + e // 2
    k_byte = (half * 512 + lane * 16 if d == 128 else lane * 16 + half * 8) + w * 4 + nib // 2
    k_bit = (nib % 2) * 4
    r, hi, word = x % 8, (x // 8) % 2, x // 16
    quad, pos = (t % 8) // 2, (t % 2) * 2 + t // 8
    v_byte = 8 * d + (word // 4) * 512 + (r * 4 + quad) * 16 + (word % 4) * 4 + pos
    v_bit = hi * 4
    tt, g = torch.meshgrid(torch.arange(16), torch.arange(d // GROUP), indexing="ij")
    k_scale = 16 * d + ((tt // 2) * (d // GROUP) + g) * 8 + (tt % 2) * 2
    return {k: v.cuda() for k, v in dict(k_byte=k_byte, k_bit=k_bit, v_byte=v_byte, v_bit=v_bit, k_scale=k_scale, v_scale=k_scale + 2 * d).items()}


def _quantise(x):
    """Codes (0 to 15), scales and minima of rows [..., d], in 32 bits."""
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    s, m = ((hi - lo) / 15).half(), lo.half()
    r = torch.where(s == 0, torch.zeros_like(lo), 1 / s.float())
    codes = ((g - m.float()[..., None]) * r[..., None]).round().clamp(0, 15)
    return codes.flatten(-2).to(torch.uint8), s, m


def _put(cache, places, slots, k, v):
    """Rows k, v [T, kv_heads, d] into the slots of the cache."""
    T, H, d = k.shape
    page = cache.shape[2] * 16
    block = (slots.long() // page * H)[:, None] + torch.arange(H, device=k.device)              # [T, H]
    base = (block * cache.shape[2] + (slots.long() % page // 16)[:, None]) * cache.shape[3]
    t = slots.long() % 16
    flat = cache.view(-1)
    for x, name in ((k, "k"), (v, "v")):
        codes, s, m = _quantise(x)
        if name == "k":          # the two codes of a byte: coordinates two apart
            pairs = codes.unflatten(-1, (-1, 2, 2, 2)).transpose(-1, -2)                          # [.., octets, 2, parity, low / high]
            both = (pairs[..., 0] | (pairs[..., 1] << 4)).flatten(-3)
            at = places["k_byte"].unflatten(-1, (-1, 2, 2, 2)).transpose(-1, -2)[..., 0].flatten(-3)
        else:                    # eight apart
            pairs = codes.unflatten(-1, (-1, 2, 8))
            both = (pairs[..., 0, :] | (pairs[..., 1, :] << 4)).flatten(-2)
            at = places["v_byte"].unflatten(-1, (-1, 2, 8))[..., 0, :].flatten(-2)
        flat[base[..., None] + at[t][:, None]] = both
        where = base[..., None] + places[name + "_scale"][t][:, None]
        for half, offset in ((s, 0), (m, 4)):
            two = half.view(torch.uint8).unflatten(-1, (-1, 2))
            flat[where + offset] = two[..., 0]
            flat[where + offset + 1] = two[..., 1]


def _get(blocks, places, d, dtype=torch.float32):
    """K and V [..., 16, d] of blocks [..., 20 d]."""
    out = []
    for name in ("k", "v"):
        at = places[name + "_byte"].flatten()
        codes = ((blocks[..., at] >> places[name + "_bit"].flatten().to(torch.uint8)) & 15).unflatten(-1, (16, -1, GROUP))
        halves = blocks.view(torch.float16)
        where = places[name + "_scale"].flatten() // 2
        s = halves[..., where].unflatten(-1, (16, -1)).to(dtype)
        m = halves[..., where + 2].unflatten(-1, (16, -1)).to(dtype)
        out.append((m[..., None] + s[..., None] * codes.to(dtype)).flatten(-2))
    return out


def _rows(cache, places, d, table, request, token):
    """K and V [T, kv_heads, d] of given tokens of given requests."""
    page = cache.shape[2] * 16
    pages = table[request, token // page].long()
    blocks = cache[pages, :, token % page // 16]                                                # [T, H, 20 d]
    t = token % 16
    out = []
    for name in ("k", "v"):
        at = places[name + "_byte"][t][:, None].expand(-1, blocks.shape[1], -1)
        codes = (blocks.gather(-1, at) >> places[name + "_bit"][t][:, None].to(torch.uint8)) & 15
        where = (places[name + "_scale"][t] // 2)[:, None].expand(-1, blocks.shape[1], -1)
        s, m = blocks.view(torch.float16).gather(-1, where).float(), blocks.view(torch.float16).gather(-1, where + 2).float()
        out.append((m[..., None] + s[..., None] * codes.unflatten(-1, (-1, GROUP)).float()).flatten(-2))
    return out


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _keys(T, H, d, gen):
    offset = torch.randn(H, d, generator=gen, device="cuda")
    return torch.randn(T, H, d, generator=gen, device="cuda") + offset


def _pages(lens, page, gen, spare=3):
    """A block table over shuffled pages, and how many pages there are."""
    need = [-(-n // page) for n in lens]
    total, width = sum(need) + spare, max(max(need), 1)
    order = torch.randperm(total, generator=gen, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, total


def _filled(case, lens, table, pages, places, gen):
    """A cache that holds keys and values of the contexts."""
    H, d, page = case["kv_heads"], case["d"], case["page"]
    cache = torch.zeros(pages, H, page // 16, 20 * d, dtype=torch.uint8, device="cuda")
    offset = torch.randn(H, d, generator=gen, device="cuda")
    step = max(1, (1 << 25) // (H * d * page))                       # pages at a time
    for p in range(0, pages, step):
        n = min(step, pages - p) * page
        slots = torch.arange(p * page, p * page + n, device="cuda")
        k = torch.randn(n, H, d, generator=gen, device="cuda") + offset
        v = torch.randn(n, H, d, generator=gen, device="cuda")
        _put(cache, places, slots, k.to(_dtype(case)), v.to(_dtype(case)))
    return cache


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] == "plan":
        rng = np.random.Generator(np.random.PCG64(seed))
        R, P = case["requests"], case["page"]
        lens = rng.integers(0, case["longest"] - case["prompt"] + 1 if case["longest"] > case["prompt"] else 1, R)
        kind = rng.random(R)
        new = np.where(kind < 0.05, -1, np.where(kind < 0.1, rng.integers(1, case["prompt"] + 1, R), 1))
        lens[(new > 1)] = rng.integers(0, 2, int((new > 1).sum())) * lens[(new > 1)]
        need = -(-lens // P)
        width = -(-case["longest"] // P) + 1
        owned = int(need.sum())
        spare = int((-(-(lens + np.maximum(new, 0)) // P) - need).sum()) + 100
        pages = R * width + 100                       # the free list has a place for every page of the cache
        order = rng.permutation(pages).astype(np.int32)
        table = np.full((R, width), -1, np.int32)
        table[np.arange(width)[None] < need[:, None]] = order[:owned]
        free = np.full(pages, -1, np.int32)
        free[:spare] = order[owned:owned + spare]     # the others belong to somebody else
        state["rows"] = _plan_rows(case)
        for name, x in dict(lengths=lens, new=new, table=table, free=free, n_free=np.array([spare])).items():
            state[name] = torch.from_numpy(x.astype(np.int32)).cuda()
        return state
    H, d, T = case["kv_heads"], case["d"], _dtype(case)
    past, new = _lengths(case)
    if case["op"] == "prompt":
        Tq, Tk = sum(new), sum(past) + sum(new)
        state["q"] = torch.randn(Tq, case["q_heads"], d, generator=gen, device="cuda").to(T)
        state["k"] = _keys(Tk, H, d, gen).to(T)
        state["v"] = torch.randn(Tk, H, d, generator=gen, device="cuda").to(T)
        state["cu_q"], state["cu_k"] = _offsets(new), _offsets([a + b for a, b in zip(past, new)])
        return state
    lens = [a + b for a, b in zip(past, new)]
    places = state["places"] = _places(d)
    state["table"], pages = _pages(lens, case["page"], gen)
    if case["op"] == "store":
        state["cache"] = torch.zeros(pages, H, case["page"] // 16, 20 * d, dtype=torch.uint8, device="cuda")
        state["k"] = _keys(case["new"], H, d, gen).to(T)
        state["v"] = torch.randn(case["new"], H, d, generator=gen, device="cuda").to(T)
        state["cu"], state["first"], state["rows"] = _offsets(new), torch.tensor(past, dtype=torch.int32, device="cuda"), case["new"]
        request = torch.repeat_interleave(torch.arange(len(new), device="cuda"), state["cu"].diff().long())
        token = torch.arange(case["new"], device="cuda") - state["cu"][request] + state["first"][request]
        state["slots"] = (state["table"][request, token // case["page"]] * case["page"] + token % case["page"]).int()
        return state
    state["cache"] = _filled(case, lens, state["table"], pages, places, gen)
    if case["op"] == "read":
        state["cu"], state["rows"] = _offsets(lens), sum(lens)
    else:
        state["q"] = torch.randn(len(lens), case["q_heads"], d, generator=gen, device="cuda").to(T)
        state["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return state


def _plan_rows(case):
    """Rows of the step's packed batch: what it may hold, whatever the step brings."""
    return max(64, case["requests"] * (1 + case["prompt"] // 10))


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _plain_plan(s):
    P, R, W, F, T = s["case"]["page"], s["table"].shape[0], s["table"].shape[1], s["free"].shape[0], s["rows"]
    lens, new = s["lengths"], s["new"]
    dev = lens.device
    have = (lens + P - 1) // P
    stays = new >= 0
    add = new.clamp(min=0)
    pages = (lens + add + P - 1) // P
    fits = stays & (pages <= W)
    released = torch.where(stays, 0, have)
    need = torch.where(fits, pages - have, 0)
    rel_end, need_end = released.cumsum(0), need.cumsum(0)
    N = s["n_free"] + rel_end[-1:]
    admitted = fits & ((need == 0) | (need_end <= N))
    given = torch.where(admitted, need, 0)
    n_free = N - given.sum()
    # the stack: free pages, then the released ones
    i = torch.arange(F, device=dev)
    j = i - s["n_free"]
    r = torch.searchsorted(rel_end, j.clamp(min=0), right=True).clamp(max=R - 1)
    p = (j - (rel_end - released)[r]).clamp(0, W - 1)
    stack = torch.where(i < s["n_free"], s["free"], s["table"][r, p])
    free = torch.where(i < n_free, stack, -1)
    # tables
    col = torch.arange(W, device=dev)[None]
    k = (need_end - need)[:, None] + col - have[:, None]
    fresh = stack[(N - 1 - k).clamp(0, F - 1)]
    table = torch.where(stays[:, None] & (col < have[:, None]), s["table"], -1)
    table = torch.where(admitted[:, None] & (col >= have[:, None]) & (col < pages[:, None]), fresh, table)
    lengths = torch.where(stays, torch.where(admitted, lens + add, lens), 0)
    zero = torch.zeros(1, dtype=torch.int32, device=dev)
    cu_new, cu_len = torch.cat([zero, add.cumsum(0)]), torch.cat([zero, lengths.cumsum(0)])
    # tokens
    row = torch.arange(T, device=dev)
    r = torch.searchsorted(cu_new[1:].contiguous(), row, right=True).clamp(max=R - 1)
    there = (row < cu_new[-1]) & admitted[r]
    pos = lens[r] + row - cu_new[r]
    page = table[r, (pos // P).clamp(0, W - 1)]
    slots = torch.where(there & (page >= 0), page * P + pos % P, -1)
    out = dict(slots=slots, positions=torch.where(there, pos, -1), cu_new=cu_new, cu_len=cu_len, lengths=lengths, table=table, free=free, n_free=n_free)
    return {name: x.int() for name, x in out.items()}


def _softmax_products(scores, seen, v):
    """softmax over the seen scores of the last axis, times v; and the log of the sum of exponentials."""
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weights = scores.sub_(top).exp_()
    total = weights.sum(-1, keepdim=True)
    out = weights @ v / torch.where(total == 0, 1.0, total)
    return out, (top + total.log()).squeeze(-1)


def _plain_attend(s):
    case = s["case"]
    R, W = s["table"].shape
    H, d, page = case["kv_heads"], case["d"], case["page"]
    blocks = s["cache"][s["table"].clamp(min=0).long()]                                          # [R, W, H, page / 16, 20 d]
    k, v = (x.permute(0, 2, 1, 3, 4, 5).reshape(R, H, W * page, d) for x in _get(blocks, s["places"], d))
    q = s["q"].float().view(R, H, -1, d)
    seen = torch.arange(W * page, device=q.device) < s["lengths"][:, None]
    out, lse = _softmax_products(q @ k.transpose(-1, -2) * (1 / math.sqrt(d)), seen[:, None, None], v)
    return out.reshape(R, -1, d).to(s["q"].dtype), lse.reshape(R, -1)


def _plain_prompt(s):
    case = s["case"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    Tq, Tk, H, d = q.shape[0], k.shape[0], case["kv_heads"], case["d"]
    rows, cols = torch.arange(Tq, device=q.device), torch.arange(Tk, device=q.device)
    rq = torch.searchsorted(s["cu_q"][1:].contiguous(), rows, right=True)
    rk = torch.searchsorted(s["cu_k"][1:].contiguous(), cols, right=True)
    # a row's distance from the end of its request against a key's
    seen = (rq[:, None] == rk) & ((s["cu_q"][rq + 1] - rows)[:, None] <= s["cu_k"][rk + 1] - cols)
    q = q.view(Tq, H, -1, d).permute(1, 2, 0, 3)
    scores = (q.reshape(H, -1, d) @ k.permute(1, 2, 0)).mul_(1 / math.sqrt(d)).view(H, -1, Tq, Tk)
    out, lse = _softmax_products(scores, seen, v.permute(1, 0, 2)[:, None])
    return out.permute(2, 0, 1, 3).reshape(Tq, -1, d).to(s["q"].dtype), lse.permute(2, 0, 1).reshape(Tq, -1)


def _plain_read(s, first=0):
    rows = torch.arange(s["rows"], device="cuda")
    r = torch.searchsorted(s["cu"][1:].contiguous(), rows, right=True)
    token = rows - s["cu"][r] + (first if isinstance(first, int) else first[r])
    k, v = _rows(s["cache"], s["places"], s["case"]["d"], s["table"], r, token)
    return k.to(_dtype(s["case"])), v.to(_dtype(s["case"]))


def _plain_store(s):
    _put(s["cache"], s["places"], s["slots"], s["k"], s["v"])
    return _plain_read(s, s["first"])


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"plan": _plain_plan, "store": _plain_store, "read": _plain_read, "attend": _plain_attend, "prompt": _plain_prompt}[op](s)
    import paper_2310_05869_b200 as ha

    if op == "plan":
        return ha.cache_plan(s["lengths"], s["new"], s["table"], s["free"], s["n_free"], s["case"]["page"], s["rows"])._asdict()
    if op == "store":
        ha.cache_store(s["cache"], s["k"], s["v"], s["slots"])
        return ha.cache_read(s["cache"], s["table"], s["cu"], s["rows"], first=s["first"], dtype=s["k"].dtype)
    if op == "read":
        return ha.cache_read(s["cache"], s["table"], s["cu"], s["rows"], dtype=_dtype(s["case"]))
    if op == "attend":
        return ha.cache_attention(s["q"], s["cache"], s["table"], s["lengths"])
    return ha.prompt_attention(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"])


def work(case):
    if case["op"] == "plan":
        R, T = case["requests"], _plan_rows(case)
        width = -(-case["longest"] // case["page"]) + 1
        pages = R * width + 100
        return {"bytes": 4 * (2 * R * width + pages + 2 * T + 5 * R), "flops": 0}
    past, new = _lengths(case)
    H, d = case["kv_heads"], case["d"]
    entry = 2 * H * d                                 # values of K and V of one token
    packed = entry * 5 // 8                           # their bytes in the cache: 4 bits, and 4 bytes for 32 of them
    if case["op"] == "store":                         # written, and read back
        return {"bytes": case["new"] * (2 * entry + 2 * packed + 2 * entry), "flops": 10 * case["new"] * entry}
    if case["op"] == "read":
        return {"bytes": case["tokens"] * (packed + 2 * entry), "flops": 2 * case["tokens"] * entry}
    hq = case["q_heads"]
    if case["op"] == "attend":
        return {"bytes": sum(past) * packed + len(past) * hq * (4 * d + 4), "flops": 4 * d * hq * sum(past)}
    pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
    return {"bytes": sum(new) * hq * (4 * d + 4) + (sum(past) + sum(new)) * 2 * entry, "flops": 4 * d * hq * pairs}


# ---- the operators' definitions in 64 bits --------------------------------------------------------------------------------
def _exact_group_values(x):
    """What the cache holds in the place of rows [T, H, d]."""
    T, H, d = x.shape
    g = x.double().reshape(T, H, d // GROUP, GROUP)
    low = g.min(-1, keepdim=True).values
    scale = ((g.max(-1, keepdim=True).values - low) / 15).to(torch.float16).double()
    low = low.to(torch.float16).double()
    code = torch.where(scale > 0, torch.round((g - low) / torch.where(scale > 0, scale, 1.0)), 0.0).clamp(0, 15)
    return (low + scale * code).reshape(T, H, d)


def _exact_context(s, r, n):
    """K and V [H, n, d] of request r's first n tokens, unpacked byte by byte."""
    cache, d, page = s["cache"], s["case"]["d"], s["case"]["page"]
    H = cache.shape[1]
    k_out, v_out = [], []
    for first in range(0, n, 1 << 14):               # so many tokens at a time
        count = min(1 << 14, n - first)
        pages = s["table"][r, first // page:-(-(first + count) // page)].long()
        b = cache[pages].transpose(0, 1).reshape(H, -1, 20 * d)                                  # [H, blocks, 20 d]
        low, high = b & 15, b >> 4
        halves = b[..., 16 * d:].contiguous().view(torch.float16).double().reshape(H, -1, 2, 8, d // GROUP, 2, 2)   # [.., k / v, pair, group, s / m, parity]
        scale = halves[..., 0, :].permute(0, 1, 2, 3, 5, 4).reshape(H, -1, 2, 16, d // GROUP, 1)
        least = halves[..., 1, :].permute(0, 1, 2, 3, 5, 4).reshape(H, -1, 2, 16, d // GROUP, 1)
        # K: 16 bytes a lane (row, octet), or 8 for either half at d = 64; bytes 0..3 of a word hold (0, 2), (4, 6), (1, 3), (5, 7) of an octet
        kn = torch.stack([low, high], -1)[..., :8 * d, :]
        if d == 128:
            kn = kn.reshape(H, -1, 2, 8, 4, 4, 4, 2)                                             # [half, row, octet, word, byte, low / high]
        else:
            kn = kn.reshape(H, -1, 8, 4, 2, 2, 4, 2).permute(0, 1, 4, 2, 3, 5, 6, 7)
        kn = kn.permute(0, 1, 2, 3, 5, 4, 6, 7).reshape(H, -1, 16, d // 32, 4, 8)                # [token, word, octet, nibble]
        kn = kn[..., [0, 4, 1, 5, 2, 6, 3, 7]].reshape(H, -1, 16, d // GROUP, GROUP)
        # V: a word holds four tokens (2c, 8 + 2c, 2c + 1, 9 + 2c) of coordinates 16 w + row (low) and 16 w + 8 + row (high)
        vn = torch.stack([low, high], -1)[..., 8 * d:16 * d, :].reshape(H, -1, d // 64, 8, 4, 4, 2, 2, 2)   # [w / 4, row, c, w % 4, parity, half, low / high]
        vn = vn.permute(0, 1, 7, 4, 6, 2, 5, 8, 3).reshape(H, -1, 16, d // GROUP, GROUP)
        for codes, which, out in ((kn, 0, k_out), (vn, 1, v_out)):
            x = least[:, :, which] + scale[:, :, which] * codes.double()
            x = x.reshape(H, -1, d)                      # from the first token of the first page on
            out.append(x[:, first % page:first % page + count])
    return torch.cat(k_out, 1), torch.cat(v_out, 1)


def _exact_rows(q, k, v, visible):
    """Attention of rows q over k, v; row i sees the first visible[i] keys."""
    d = q.shape[-1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full(q.shape[:-1], -math.inf, dtype=torch.float64, device=q.device)
    step = max(1, (1 << 27) // max(1, k.shape[0]))
    for i in range(0, q.shape[0], step):
        z = q[i:i + step] @ k.T / math.sqrt(d)
        z = torch.where(torch.arange(k.shape[0], device=q.device) < visible[i:i + step, None], z, -math.inf)
        there = visible[i:i + step] > 0
        lse[i:i + step] = torch.logsumexp(z, -1)
        w = torch.softmax(z, -1)
        out[i:i + step] = torch.where(there[:, None], torch.where(there[:, None], w, 0.0) @ v, 0.0)
    return out, lse


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    past, new = _lengths(case)
    if case["op"] == "store":
        return _exact_group_values(s["k"]), _exact_group_values(s["v"])
    if case["op"] == "read":
        parts = [_exact_context(s, r, n) for r, n in enumerate(past)]
        return tuple(torch.cat([p[i].transpose(0, 1) for p in parts]) for i in (0, 1))
    H, hq = case["kv_heads"], case["q_heads"]
    G = hq // H
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    if case["op"] == "attend":
        for r, n in enumerate(past):
            if n:
                k, v = _exact_context(s, r, n)
                q = s["q"][r].double().view(H, G, -1)
                z = q @ k.transpose(1, 2) / math.sqrt(case["d"])
                lse[r] = torch.logsumexp(z, -1).flatten()
                out[r] = (torch.softmax(z, -1) @ v).flatten(0, 1)
        return out, lse
    q0 = k0 = 0
    for p, n in zip(past, new):
        visible = torch.arange(p + 1, p + n + 1, device="cuda")
        for h in range(hq):
            k, v = (s[x][k0:k0 + p + n, h // G].double() for x in ("k", "v"))
            out[q0:q0 + n, h], lse[q0:q0 + n, h] = _exact_rows(s["q"][q0:q0 + n, h].double(), k, v, visible)
        q0, k0 = q0 + n, k0 + p + n
    return out, lse
