"""Performance cases of the operators by which a server of long contexts adds to a paged 4-bit cache and keeps it within bounds.

Four operators, two to four cases each:

  chunk    attention of some new tokens a request over the cache (their own keys are in it): parts of prompts, drafted tokens
  weights  attention weight that every cached token gets from such rows, added to what it got before
  pages    new pages for what stays of requests that have grown too long, their old pages back on the stack
  evict    the tokens of most weight (and the first and the last ones) of such requests, moved to those pages, for every key head by itself;
           read back, as the values that the cache stands for

Head counts and widths: 32 heads of 64 or 128 as in the benchmark configurations, with as many key / value heads, a quarter of
them, or two.  The cache's pages have 64 tokens unless a case says otherwise.

Layout of the cache, [pages, kv_heads, page / 16, 20 d] bytes: blocks of 16 tokens of one head, in each 8 d bytes of K codes, 8 d of V
codes, then scales and minima of the groups of 32 coordinates (fp16), 2 d bytes for K, 2 d for V.  A value is minimum + scale * code.

Inputs are synthetic, made on the GPU: queries and values N(0, 1), keys N(0, 1) around an offset per channel (as keys have), accumulated
weights with a long tail."""
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
        # Four drafted tokens for each of a few chats: latency.
        "chunk_draft_8": _case("chunk", requests=8, new=32, longest=1500, q_heads=32, kv_heads=8, d=128, page=64, dtype="bf16"),
        # Drafted tokens over the headline context, as many key heads as query heads: the cache is read once.
        "chunk_draft_131k": _case("chunk", requests=2, new=16, longest=131000, q_heads=32, kv_heads=32, d=64, page=64, dtype="fp16"),
        # The next parts of prompts of different lengths, side by side, none of them a multiple of anything.
        "chunk_parts_1500": _case("chunk", requests=5, new=1501, longest=5000, q_heads=32, kv_heads=32, d=64, page=16, dtype="fp16"),
        # A part of one long prompt.
        "chunk_2k_32k": _case("chunk", requests=1, new=2048, longest=30720, q_heads=32, kv_heads=8, d=128, page=64, dtype="bf16"),
        # What a decode step of a batch adds, one token a request.
        "weights_decode_64": _case("weights", requests=64, new=64, longest=8192, q_heads=32, kv_heads=8, d=128, page=64, dtype="bf16"),
        # The same for a few chats: latency.
        "weights_chats_4": _case("weights", requests=4, new=4, longest=600, q_heads=32, kv_heads=2, d=128, page=64, dtype="fp16"),
        # What a part of a prompt adds.
        "weights_part_1k": _case("weights", requests=2, new=1025, longest=32000, q_heads=32, kv_heads=32, d=64, page=64, dtype="bf16"),
        # A batch of which about half has grown too long.
        "pages_256": _case("pages", requests=256, longest=8192, page=64),
        # The most that is looked at in one step.
        "pages_1024": _case("pages", requests=1024, longest=131072, page=64),
        # Chats that are cut to a window: latency.
        "evict_chats_4": _case("evict", requests=4, longest=1200, keep=256, kv_heads=2, d=128, page=16, dtype="bf16"),
        # A batch, cut to a quarter of the longest.
        "evict_batch_32": _case("evict", requests=32, longest=8192, keep=2048, kv_heads=8, d=128, page=64, dtype="bf16"),
        # Long contexts, cut to a sixteenth.
        "evict_131k": _case("evict", requests=2, longest=131072, keep=8192, kv_heads=32, d=64, page=64, dtype="fp16"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def draw(rng):
    def span(lo, hi):              # log-uniform, both ends included
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    def heads():
        return rng.choice([(32, 32, 64), (32, 8, 128), (32, 2, 128), (16, 2, 128), (32, 8, 64), (12, 12, 64), (28, 4, 128), (9, 3, 64)])

    op = rng.choice(["chunk", "chunk", "chunk", "weights", "weights", "pages", "evict", "evict"])
    hq, hkv, d = heads()
    page, dtype = rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "fp16"])
    longest = span(100, 131000)
    if op == "pages":
        case = _case(op, requests=span(1, 1024), longest=longest, page=page)
    elif op == "evict":
        case = _case(op, requests=span(1, 64), longest=longest, keep=span(32, max(33, longest // 2)), kv_heads=hkv, d=d, page=page, dtype=dtype)
    else:
        new = span(1, 2048)
        case = _case(op, requests=min(new, span(1, 64)), new=new, longest=longest, q_heads=hq, kv_heads=hkv, d=d, page=page, dtype=dtype)
    most = [_cost(c) for c in listed() if c["op"] == op]
    while any(x > max(y) for x, y in zip(_cost(case), zip(*most))):
        case["longest"] = case["longest"] * 3 // 4
        if "keep" in case:
            case["keep"] = max(1, min(case["keep"], case["longest"] // 2))
        elif "new" in case and rng.random() < 0.5:
            case["new"] = max(1, case["new"] * 3 // 4)
            case["requests"] = min(case["requests"], case["new"])
    return case


def _cost(case):
    """Work, and the scores of a plain form, whose requests are as long as the longest."""
    w, scores = work(case), 0
    if "new" in case:
        past, new = _lengths(case)
        scores = len(past) * max(new) * case["q_heads"] * max(p + n for p, n in zip(past, new))
    return w["flops"], w["bytes"], scores


def _dtype(case):
    return {"bf16": torch.bfloat16, "fp16": torch.float16}[case["dtype"]]


# ---- lengths: made from the case alone, so that the work of a pass can be told without its inputs -----------------------
def _lengths(case):
    """(tokens that are cached before, new tokens) of every request; evict: (cached, those that stay)."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    R = case["requests"]
    past = [rng.randint(0, case["longest"]) for _ in range(R)]
    past[0] = case["longest"]
    if R > 8:
        past[1], past[2] = 0, 1
    if case["op"] == "evict":
        return past, [min(n, case["keep"]) for n in past]
    weights = [rng.random() + 0.5 for _ in range(R)]                 # a token at least each
    scale = (case["new"] - R) / sum(weights)
    new = [1 + int(w * scale) for w in weights]
    new[-1] += case["new"] - sum(new)
    return past, new


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


def _blocks(k, v, places):
    """Bytes [n, 20 d] of blocks that hold k, v [n, 16, d]."""
    n, _, d = k.shape
    out = torch.zeros(n, 20 * d, dtype=torch.uint8, device=k.device)
    for x, name in ((k, "k"), (v, "v")):
        g = x.float().unflatten(-1, (-1, GROUP))
        lo, hi = g.amin(-1), g.amax(-1)
        s, m = ((hi - lo) / 15).half(), lo.half()
        r = torch.where(s == 0, torch.zeros_like(lo), 1 / s.float())
        codes = ((g - m.float()[..., None]) * r[..., None]).round().clamp(0, 15).flatten(-2).to(torch.uint8)
        for bit in (0, 4):                                # the two codes of a byte
            here = places[name + "_bit"] == bit
            out[:, places[name + "_byte"][here]] |= codes[:, here] << bit
        for half, offset in ((s, 0), (m, 4)):
            two = half.view(torch.uint8).unflatten(-1, (-1, 2))
            at = places[name + "_scale"] + offset
            out[:, at], out[:, at + 1] = two[..., 0], two[..., 1]
    return out


def _values(blocks, places, d):
    """K and V [..., 16, d] of blocks [..., 20 d], in 32 bits."""
    out = []
    for name in ("k", "v"):
        at = places[name + "_byte"].flatten()
        codes = ((blocks[..., at] >> places[name + "_bit"].flatten().to(torch.uint8)) & 15).unflatten(-1, (16, -1, GROUP))
        halves = blocks.view(torch.float16)
        where = places[name + "_scale"].flatten() // 2
        s = halves[..., where].unflatten(-1, (16, -1)).float()
        m = halves[..., where + 2].unflatten(-1, (16, -1)).float()
        out.append((m[..., None] + s[..., None] * codes.float()).flatten(-2))
    return out


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _pages(lens, page, gen, spare):
    """A block table over shuffled pages, the pages that are left, and how many there are."""
    need = [-(-n // page) for n in lens]
    total, width = sum(need) + spare, max(max(need), 1)
    order = torch.randperm(total, generator=gen, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, order[at:], total


def _filled(case, pages, places, gen):
    """A cache that holds keys and values in all of its places."""
    H, d, page = case["kv_heads"], case["d"], case["page"]
    cache = torch.empty(pages, H, page // 16, 20 * d, dtype=torch.uint8, device="cuda")
    offset = torch.randn(H, 1, d, generator=gen, device="cuda")
    step = max(1, (1 << 25) // (H * d * page))                       # pages at a time
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k = torch.randn(n, H, page, d, generator=gen, device="cuda") + offset
        v = torch.randn(n, H, page, d, generator=gen, device="cuda")
        k, v = (x.to(_dtype(case)).view(-1, 16, d) for x in (k, v))
        cache[p:p + n] = _blocks(k, v, places).view(n, H, page // 16, 20 * d)
    return cache


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    state = {"case": case}
    if case["op"] == "pages":
        rng = np.random.Generator(np.random.PCG64(seed))
        R, P = case["requests"], case["page"]
        lens = rng.integers(0, case["longest"] + 1, R)
        keep = np.where(rng.random(R) < 0.1, -1, case["longest"] // 2)               # (-1: this one stays as it is)
        need = -(-lens // P)
        width = -(-case["longest"] // P)
        owned, spare = int(need.sum()), R * (-(-case["longest"] // 2 // P)) // 3 + 3   # not enough for all of them now and then
        pages = R * width + spare
        order = rng.permutation(pages).astype(np.int32)
        table = np.full((R, width), -1, np.int32)
        table[np.arange(width)[None] < need[:, None]] = order[:owned]
        free = np.full(pages, -1, np.int32)
        free[:spare] = order[owned:owned + spare]                                      # the others belong to somebody else
        for name, x in dict(lengths=lens, keep=keep, table=table, free=free, n_free=np.array([spare])).items():
            state[name] = torch.from_numpy(x.astype(np.int32)).cuda()
        return state
    H, d, P = case["kv_heads"], case["d"], case["page"]
    past, new = _lengths(case)
    lens = past if case["op"] == "evict" else [a + b for a, b in zip(past, new)]
    places = state["places"] = _places(d)
    room = sum(-(-n // P) for m, n in zip(past, new) if n < m) if case["op"] == "evict" else 0
    state["table"], left, pages = _pages(lens, P, gen, 3 + room)
    state["cache"] = _filled(case, pages, places, gen)
    state["lengths"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cap = state["table"].shape[1] * P
    if case["op"] != "chunk":
        there = torch.arange(cap, device="cuda") < state["lengths"][:, None, None]
        weights = torch.randn(len(lens), H, cap, generator=gen, device="cuda").mul_(2).exp_()
        few = torch.rand(len(lens), H, cap, generator=gen, device="cuda") < 0.05         # tokens that nobody looked at
        state["weights"] = torch.where(there & ~few, weights, 0.0)
        del weights, few
    if case["op"] == "evict":
        keep = torch.tensor(new, dtype=torch.int32, device="cuda")
        need = torch.where(keep < state["lengths"], (keep + P - 1) // P, 0)
        to = torch.full_like(state["table"], -1)
        col = torch.arange(to.shape[1], device="cuda")
        at = ((need.cumsum(0) - need)[:, None] + col).clamp(max=max(left.numel() - 1, 0))
        state["to"] = torch.where((keep < state["lengths"])[:, None], torch.where(col < need[:, None], left[at], -1), state["table"]).int()
        state["kept"], state["cu"], state["rows"] = keep, _offsets(new), sum(new)
        state["recent"], state["first"] = case["keep"] // 4, 4
        return state
    state["q"] = torch.randn(sum(new), case["q_heads"], d, generator=gen, device="cuda").to(_dtype(case))
    state["cu"], state["decay"] = _offsets(new), 0.97
    if case["op"] == "weights":
        state["lse"] = _lse(_scores(state))[_inside(state)]
    return state


# ---- plain forms ---------------------------------------------------------------------------------------------------------
def _inside(s):
    """Which rows of the requests' queries, padded to the most that one has, are there [R, n]."""
    count = s["cu"].diff()
    return torch.arange(max(_lengths(s["case"])[1]), device="cuda") < count[:, None]


def _context(s):
    """K and V [R, H, cap, d] of the tables' pages."""
    R, W = s["table"].shape
    blocks = s["cache"][s["table"].clamp(min=0).long()]                                          # [R, W, H, page / 16, 20 d]
    return (x.permute(0, 2, 1, 3, 4, 5).reshape(R, blocks.shape[2], -1, s["case"]["d"]) for x in _values(blocks, s["places"], s["case"]["d"]))


def _scores(s, k=None):
    """[R, n, H, G, cap], minus infinity where a row does not see a key."""
    k = next(_context(s)) if k is None else k
    R, H, cap, d = k.shape
    inside = _inside(s)
    n = inside.shape[1]
    at = (s["cu"][:-1, None] + torch.arange(n, device="cuda")).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at.long()].float().view(R, n, H, -1, d).permute(0, 2, 1, 3, 4)                   # [R, H, n, G, d]
    z = (q.reshape(R, H, -1, d) @ k.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(R, H, n, -1, cap)
    last = s["lengths"][:, None] - s["cu"].diff()[:, None] + torch.arange(n, device="cuda")       # last key that a row sees
    seen = (torch.arange(cap, device="cuda") <= last[..., None]) & inside[..., None]
    return z.masked_fill_(~seen[:, None, :, None], -math.inf).permute(0, 2, 1, 3, 4)


def _lse(z):
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    return ((z - top).exp_().sum(-1, keepdim=True).log() + top).squeeze(-1).flatten(2)           # [R, n, Hq]


def _plain_chunk(s):
    k, v = _context(s)
    z = _scores(s, k)
    R, n, H, G, cap = z.shape
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    out = (z.permute(0, 2, 1, 3, 4).reshape(R, H, n * G, cap) @ v).view(R, H, n, G, -1).transpose(1, 2) / torch.where(total == 0, 1.0, total)
    inside = _inside(s)
    return out.flatten(2, 3)[inside].to(s["q"].dtype), (top + total.log()).squeeze(-1).flatten(2)[inside]


def _plain_weights(s):
    z = _scores(s)
    R, n, H, G, cap = z.shape
    at = (s["cu"][:-1, None] + torch.arange(n, device="cuda")).clamp(max=s["q"].shape[0] - 1)
    lse = s["lse"][at.long()].view(R, n, H, G, 1)
    got = z.sub_(lse).exp_().sum((1, 3))                                                          # [R, H, cap]
    before = s["lengths"] - s["cu"].diff()
    old = torch.arange(cap, device="cuda") < before[:, None, None]
    return torch.where(old, s["decay"] * s["weights"], 0.0) + got


def _plain_pages(s):
    P, (R, W), F = s["case"]["page"], s["table"].shape, s["free"].shape[0]
    lens, dev = s["lengths"], s["table"].device
    have = (lens + P - 1) // P
    wants = (s["keep"] >= 0) & (s["keep"] < lens)
    need = torch.where(wants, (s["keep"] + P - 1) // P, 0)
    need_end = need.cumsum(0)
    moved = wants & ((need == 0) | (need_end <= s["n_free"]))
    given = torch.where(moved, need, 0).sum()
    released = torch.where(moved, have, 0)
    rel_end = released.cumsum(0)
    left = s["n_free"] - given
    i = torch.arange(F, device=dev)
    r = torch.searchsorted(rel_end, (i - left).clamp(min=0), right=True).clamp(max=R - 1)
    p = (i - left - (rel_end - released)[r]).clamp(0, W - 1)
    n_free = left + rel_end[-1]
    free = torch.where(i < left, s["free"], torch.where(i < n_free, s["table"][r, p], -1))
    col = torch.arange(W, device=dev)[None]
    fresh = s["free"][(s["n_free"] - 1 - (need_end - need)[:, None] - col).clamp(0, F - 1)]
    table = torch.where(moved[:, None], torch.where(col < need[:, None], fresh, -1), torch.where(col < have[:, None], s["table"], -1))
    return {name: x.int() for name, x in dict(lengths=torch.where(moved, s["keep"], lens), table=table, free=free, n_free=n_free).items()}


def _plain_evict(s):
    w, lens, keep = s["weights"], s["lengths"][:, None, None], s["kept"][:, None, None]
    R, H, cap = w.shape
    P, t = s["case"]["page"], torch.arange(cap, device=w.device)
    recent = torch.minimum(keep, torch.tensor(s["recent"], device=w.device))
    first = torch.minimum(keep - recent, torch.tensor(s["first"], device=w.device))
    always = (t < first) | (t >= lens - recent)
    rank = torch.where(t < lens, torch.where(always, math.inf, w), -1.0)
    order = torch.sort(rank, dim=-1, descending=True, stable=True).indices
    chosen = torch.zeros(R, H, cap, dtype=torch.bool, device=w.device).scatter_(-1, order, (t < keep).expand(R, H, -1))
    kept = torch.where(chosen, t, cap).sort(-1).values                                            # the tokens that stay, in order
    there, moved = t < keep, keep < lens
    at = torch.where(there, kept, 0)
    weights = torch.where(moved, torch.where(there, w.gather(-1, at), 0.0), w)
    kept = torch.where(moved & there, kept, -1).int()
    # every kept token of every head: codes, scales and minima go from place to place as they are
    r, h, j = (moved & there).expand(R, H, -1).nonzero(as_tuple=True)
    src = kept[r, h, j].long()
    flat, S = s["cache"].view(-1), P // 16
    from_, to = (((tab[r, x // P].long() * H + h) * S + x % P // 16) * s["cache"].shape[3] for tab, x in ((s["table"], src), (s["to"], j)))
    pl = s["places"]
    k_from, k_to = (base[:, None] + pl["k_byte"][x % 16] for base, x in ((from_, src), (to, j)))
    low = pl["k_bit"][0] == 0                                                                     # (the nibble of a coordinate does not depend on the token)
    codes = flat[k_from[:, low]] & 15, flat[k_from[:, ~low]] & 240
    flat[k_to[:, low]] = codes[0]
    flat[k_to[:, ~low]] |= codes[1]
    v_from, v_to = (base[:, None] + pl["v_byte"][x % 16][:, pl["v_bit"][0] == 0] for base, x in ((from_, src), (to, j)))
    flat[v_to] = flat[v_from]
    for name in ("k_scale", "v_scale"):
        for byte in (0, 1, 4, 5):
            flat[to[:, None] + pl[name][j % 16] + byte] = flat[from_[:, None] + pl[name][src % 16] + byte]
    return weights, kept, *_plain_read(s)


def _plain_read(s):
    """K and V [rows, H, d] of the tokens that stay, as the new pages hold them."""
    P, d = s["case"]["page"], s["case"]["d"]
    rows = torch.arange(s["rows"], device="cuda")
    r = torch.searchsorted(s["cu"][1:].contiguous(), rows, right=True)
    token = rows - s["cu"][r]
    blocks = s["cache"][s["to"][r, token // P].long(), :, token % P // 16]                        # [T, H, 20 d]
    t, out = token % 16, []
    for name in ("k", "v"):
        at = s["places"][name + "_byte"][t][:, None].expand(-1, blocks.shape[1], -1)
        codes = (blocks.gather(-1, at) >> s["places"][name + "_bit"][t][:, None].to(torch.uint8)) & 15
        where = (s["places"][name + "_scale"][t] // 2)[:, None].expand(-1, blocks.shape[1], -1)
        sc, m = blocks.view(torch.float16).gather(-1, where).float(), blocks.view(torch.float16).gather(-1, where + 2).float()
        out.append((m[..., None] + sc[..., None] * codes.unflatten(-1, (-1, GROUP)).float()).flatten(-2).to(_dtype(s["case"])))
    return out


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"chunk": _plain_chunk, "weights": _plain_weights, "pages": _plain_pages, "evict": _plain_evict}[op](s)
    import paper_2310_05869_b200 as ha

    if op == "chunk":
        return ha.cache_chunk_attention(s["q"], s["cache"], s["table"], s["lengths"], s["cu"])
    if op == "weights":
        return ha.cache_weights(s["q"], s["cache"], s["table"], s["lengths"], s["lse"], s["cu"], weights=s["weights"], decay=s["decay"])
    if op == "pages":
        return ha.cache_evict_plan(s["lengths"], s["keep"], s["table"], s["free"], s["n_free"], s["case"]["page"])._asdict()
    weights, kept = ha.cache_evict(s["cache"], s["weights"], s["table"], s["lengths"], s["to"], s["kept"], recent=s["recent"], first=s["first"])
    return weights, kept, *ha.cache_read(s["cache"], s["to"], s["cu"], s["rows"], dtype=_dtype(s["case"]))


def work(case):
    if case["op"] == "pages":
        R, width = case["requests"], -(-case["longest"] // case["page"])
        pages = R * width + R * (-(-case["longest"] // 2 // case["page"])) // 3 + 3
        return {"bytes": 4 * (2 * R * width + 2 * pages + 3 * R), "flops": 0}
    past, new = _lengths(case)
    H, d, P = case["kv_heads"], case["d"], case["page"]
    packed = 2 * H * d * 5 // 8                       # bytes of a token's K and V in the cache: 4 bits, and 4 bytes for 32 of them
    if case["op"] == "evict":
        cap = max(1, max(-(-n // P) for n in past)) * P
        moved = sum(n for m, n in zip(past, new) if n < m)
        # weights in and out, the kept tokens' places, what is moved read and written, and all that stays read back
        return {"bytes": H * (4 * sum(past) + 8 * cap * len(past)) + moved * 2 * packed + sum(new) * (packed + 4 * H * d), "flops": 0}
    hq = case["q_heads"]
    lens = [a + b for a, b in zip(past, new)]
    pairs = sum(n * p + n * (n + 1) // 2 for p, n in zip(past, new))
    if case["op"] == "weights":
        cap = max(-(-n // P) for n in lens) * P
        return {"bytes": sum(lens) * packed // 2 + sum(new) * hq * (2 * d + 4) + 4 * H * (sum(past) + cap * len(past)), "flops": 2 * d * hq * pairs}
    return {"bytes": sum(lens) * packed + sum(new) * hq * (4 * d + 4), "flops": 4 * d * hq * pairs}


# ---- the operators' definitions in 64 bits --------------------------------------------------------------------------------
def _exact_context(s, table, r, n):
    """K and V [H, n, d] of request r's first n tokens in the pages of `table`, unpacked byte by byte."""
    cache, d, page = s["cache"], s["case"]["d"], s["case"]["page"]
    H = cache.shape[1]
    k_out, v_out = [], []
    for first in range(0, n, 1 << 14):               # so many tokens at a time
        count = min(1 << 14, n - first)
        pages = table[r, first // page:-(-(first + count) // page)].long()
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


def _exact_evict(s, past, new):
    weights = s["weights"].double()
    R, H, cap = weights.shape
    out, kept, ks, vs = weights.clone(), [], [], []
    for r, (n, stay) in enumerate(zip(past, new)):
        if n == 0:
            continue
        k, v = _exact_context(s, s["table"], r, n)
        if stay < n:
            recent = min(s["recent"], stay)
            first = min(s["first"], stay - recent)
            middle = weights[r, :, first:n - recent]
            best = torch.argsort(-middle, dim=-1, stable=True)[:, :stay - recent - first] + first
            ends = torch.cat([torch.arange(first), torch.arange(n - recent, n)]).cuda().expand(H, -1)
            at = torch.cat([best, ends], -1).sort(-1).values                                      # [H, stay]
            out[r] = 0
            out[r, :, :stay] = weights[r].gather(1, at)
            k, v = (x.gather(1, at[..., None].expand(-1, -1, x.shape[-1])) for x in (k, v))
        ks.append(k.transpose(0, 1))
        vs.append(v.transpose(0, 1))
    return out, None, torch.cat(ks), torch.cat(vs)


def exact(case, seed):
    if case["op"] == "pages":
        return None
    s = prepare(case, seed)
    past, new = _lengths(case)
    if case["op"] == "evict":
        return _exact_evict(s, past, new)
    H, hq, d = case["kv_heads"], case["q_heads"], case["d"]
    G = hq // H
    q = s["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    sums = torch.zeros(len(past), H, s["table"].shape[1] * case["page"], dtype=torch.float64, device="cuda")
    first = 0
    for r, (p, n) in enumerate(zip(past, new)):
        k, v = _exact_context(s, s["table"], r, p + n)
        if case["op"] == "weights":
            sums[r, :, :p] = s["decay"] * s["weights"][r, :, :p].double()
        step = max(1, (1 << 26) // (hq * (p + n)))
        for i in range(0, n, step):
            rows = slice(first + i, first + min(n, i + step))
            x = q[rows].view(-1, H, G, d).permute(1, 0, 2, 3)                                     # [H, rows, G, d]
            z = torch.einsum("hngd,hkd->hngk", x, k) / math.sqrt(d)
            hidden = torch.arange(p + n, device="cuda") > torch.arange(p + i, p + i + x.shape[1], device="cuda")[:, None]
            z = z.masked_fill(hidden[None, :, None], -math.inf)
            if case["op"] == "weights":
                have = s["lse"][rows].double().view(-1, H, G).permute(1, 0, 2)[..., None]
                sums[r, :, :p + n] += torch.exp(z - have).sum((1, 2))
            else:
                lse[rows] = torch.logsumexp(z, -1).permute(1, 0, 2).flatten(1)
                out[rows] = torch.einsum("hngk,hkd->nhgd", torch.softmax(z, -1), v).flatten(1, 2)
        first += n
    return sums if case["op"] == "weights" else (out, lse)
