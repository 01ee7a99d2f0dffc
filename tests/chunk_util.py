"""Caches with known contents, and plain statements (64 bits) of the operators that add to a cache and keep it within bounds.  Written from the definitions in
include/hyperattn.h."""
import math

import numpy as np
import torch

import paper_2310_05869_b200 as ha
import serving_util as SU

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
JUNK = 0xFF            # what places without tokens hold: NaN scales and minima


def filled(lens, kv_heads, d, page, dtype=torch.bfloat16, seed=0, width=None, spare=5, k_scale=1.0, v_scale=1.0, put=None):
    """A cache with `lens` tokens of every request in shuffled pages: cache, table, and what it holds, K and V [sum(lens), kv_heads, d] in 64 bits.  put(k, v): changes
    the rows that are stored."""
    gen = torch.Generator("cuda").manual_seed(seed)
    need = [-(-n // page) for n in lens]
    width = width or max(max(need), 1)
    pages = sum(need) + spare
    cache = ha.cache_pages(pages, kv_heads, d, page)
    cache.fill_(JUNK)
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    T = sum(lens)
    k = ((torch.randn(T, kv_heads, d, generator=gen, device="cuda") + torch.randn(kv_heads, d, generator=gen, device="cuda")) * k_scale).to(dtype)
    v = (torch.randn(T, kv_heads, d, generator=gen, device="cuda") * v_scale).to(dtype)
    if put:
        put(k, v)
    slots = [int(table[r, t // page]) * page + t % page for r, n in enumerate(lens) for t in range(n)] if T < 5000 else None
    if slots is None:
        t = torch.cat([torch.arange(n, device="cuda") for n in lens])
        r = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), torch.tensor(lens, device="cuda"))
        slots = table[r, t // page] * page + t % page
    ha.cache_store(cache, k, v, torch.as_tensor(slots, dtype=torch.int32, device="cuda").contiguous())
    held = [torch.from_numpy(SU.held(x.float().cpu().numpy())).double().cuda() if T else x.double() for x in (k, v)]
    return cache, table, *held


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(counts):
    return ints([0] + list(np.cumsum(counts)))


def rows_of(q, k, seen_upto, there, scale=None):
    """Scores [n, G, m] (natural units, -inf where unseen) of q [n, G, d] over k [m, d]; and the largest scale sum |q k| of every row."""
    scale = scale or 1 / math.sqrt(q.shape[-1])
    z = torch.einsum("ngd,md->ngm", q, k) * scale
    size = (torch.einsum("ngd,md->ngm", q.abs(), k.abs()) * scale).nan_to_num(nan=0.0, posinf=0.0)      # (of numbers)
    seen = (torch.arange(k.shape[0], device=q.device) < seen_upto[:, None]) & there
    return torch.where(seen[:, None], z, -math.inf), torch.where(seen[:, None], size, 0.0).amax(-1) if k.shape[0] else z.new_zeros(z.shape[:2]), seen


def visible(n, length, causal):
    last = torch.arange(length - n + 1, length + 1, device="cuda").clamp(0, length)
    return last if causal else torch.full((n,), length, device="cuda")


def attention(q, k, v, lens, counts, causal=True, scale=None, there=None):
    """out, lse [T, Hq, (d)], and the bounds' ingredients: sum p |v|, the same with the largest |v| of its group of 32, and the largest scale sum |q k|.  k, v: rows of all requests, one after the other; there [sum(lens)]: is a token's page one."""
    T, Hq, d = q.shape
    H = k.shape[1]
    G = Hq // H
    out, mass, coarse = q.new_zeros(T, Hq, d), q.new_zeros(T, Hq, d), q.new_zeros(T, Hq, d)
    lse, size = q.new_full((T, Hq), -math.inf), q.new_zeros(T, Hq)
    q0 = k0 = 0
    for n, m in zip(counts, lens):
        ok = torch.ones(m, dtype=torch.bool, device="cuda") if there is None else there[k0:k0 + m]
        for h in range(H):
            if n == 0 or m == 0:
                continue
            hs = slice(h * G, h * G + G)
            kk, vv = k[k0:k0 + m, h], v[k0:k0 + m, h]
            step = max(1, (1 << 26) // (G * m))
            for a in range(0, n, step):
                b = min(n, a + step)
                z, s, seen = rows_of(q[q0 + a:q0 + b, hs], kk, visible(n, m, causal)[a:b], ok, scale)
                top = z.amax(-1, keepdim=True)
                w = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
                total = w.sum(-1, keepdim=True)
                none = total == 0
                p = torch.where(none, 0.0, w / torch.where(none, 1.0, total))
                rows = slice(q0 + a, q0 + b)
                nan = torch.isnan(vv)
                clean = torch.where(nan, 0.0, vv)
                o = p @ clean
                sees_nan = (seen.double() @ nan.double() > 0)[:, None].expand_as(o)
                out[rows, hs] = torch.where(sees_nan & ~none, math.nan, o)
                mass[rows, hs] = p @ clean.abs()
                coarse[rows, hs] = p @ clean.abs().unflatten(-1, (-1, SU.GROUP)).amax(-1, keepdim=True).expand(-1, -1, SU.GROUP).flatten(-2)
                lse[rows, hs] = (top + total.log()).squeeze(-1)
                size[rows, hs] = s
        q0 += n
        k0 += m
    return out, lse, (mass, coarse), size


def check_attention(got, want, dtype, keys, rows):
    """Against the bounds that the header's roundings add up to.  Scores: the products of exact operands are summed in fp32, at most 40 sums that lose 2^-23 of the partial sum (at
    most `size`) each: 2^-17 size.  Weights: that, 2.7e-6 of an exponential, 2^-11 as fp16; values once 2^-11 as fp16; the sum over keys 2^-23 for every 16 of them, and as many again where parts are
    joined; the result's own type (fp16 numbers below 2^-14 are multiples of 2^-24, so that half a step is 2^-25 there, whatever the size of the result).  A value is
    minimum + scale * code, two terms that may each be twice the group's largest value while the value is nearly nothing: with weights times scales as two fp16 numbers (2^-22) and the minima
    apart, and in what the sums over keys lose, it is those terms that count."""
    (out, lse), (o, l, (mass, coarse), size) = got, want
    rows = slice(0, rows)
    out, lse, o, l, mass, coarse, size = out[rows].double(), lse[rows].double(), o[rows], l[rows], mass[rows], coarse[rows], size[rows]
    score = 2.0 ** -17 * size + 2.0 ** -17
    assert torch.equal(torch.isnan(lse), torch.isnan(l)) and torch.equal(lse == -math.inf, l == -math.inf)
    fine = torch.isfinite(l)
    err = torch.where(fine, (lse - l).abs(), 0.0)
    assert bool((err <= score + 2.0 ** -23 * torch.where(fine, l.abs(), 0.0))[fine].all()), float((err / score)[fine].max())
    assert torch.equal(torch.isnan(out), torch.isnan(o))
    bound = HALF_STEP[dtype] * o.abs() + (2 * 2.0 ** -11 * 1.01 + 2 * score)[..., None] * mass + (4 * 2.0 ** -22 + 4 * (keys / 16 + 2) * 2.0 ** -23) * coarse + 2.0 ** -25 * coarse.amax(-1, keepdim=True) + (2.0 ** -25 if dtype is torch.float16 else 1e-37)
    bad = (out - o).abs() > bound
    assert not bool(bad.any()), float(((out - o).abs() / bound)[torch.isfinite(o)].max())


def weights(q, k, lens, counts, lse, before=None, decay=1.0, causal=True, scale=None, cap=None, there=None):
    """The weights and the bounds of their errors [R, H, cap]."""
    T, Hq, d = q.shape
    H, R = k.shape[1], len(lens)
    G = Hq // H
    w, bound = torch.zeros(R, H, cap, dtype=torch.float64, device="cuda"), torch.zeros(R, H, cap, dtype=torch.float64, device="cuda")
    lse = lse.double()
    q0 = k0 = 0
    for r, (n, m) in enumerate(zip(counts, lens)):
        old = max(m - n, 0)
        if before is not None:
            w[r, :, :old] = decay * before[r, :, :old].double()
            bound[r, :, :old] = 2.0 ** -23 * w[r, :, :old].abs()
        ok = torch.ones(m, dtype=torch.bool, device="cuda") if there is None else there[k0:k0 + m]
        for h in range(H):
            if n == 0 or m == 0:
                continue
            hs = slice(h * G, h * G + G)
            step = max(1, (1 << 26) // (G * m))
            for a in range(0, n, step):
                b = min(n, a + step)
                z, s, seen = rows_of(q[q0 + a:q0 + b, hs], k[k0:k0 + m, h], visible(n, m, causal)[a:b], ok, scale)
                have = lse[q0 + a:q0 + b, hs]
                p = torch.where(seen[:, None] & (have != -math.inf)[..., None], torch.exp(z - have[..., None]), 0.0)
                # a score as in check_attention, its difference to the log-sum-exp (2^-22 of either), the exponential, the sum over rows in fp32 (2^-24 each)
                each = 2.0 ** -17 * s + 2.0 ** -21 * torch.where(torch.isfinite(have), have.abs(), 0.0) + 2.0 ** -17 + 2.0 ** -24 * n * G
                w[r, h, :m] += p.sum((0, 1))
                bound[r, h, :m] += (p * each[..., None]).sum((0, 1)) + 2.0 ** -126 * n * G
        q0 += n
        k0 += m
    return w, bound + 2.0 ** -23 * w.abs()


def evict(weights, lens, keep, recent, first):
    """Which tokens stay, [R][H] lists (None: the request is not cut)."""
    out = []
    for r, (m, n) in enumerate(zip(lens, keep)):
        n = max(min(n, m), 0)
        if n >= m:
            out.append(None)
            continue
        last = min(recent, n)
        begin = min(first, n - last)
        heads = []
        for h in range(weights.shape[1]):
            w = weights[r, h, :m].astype(np.float64)
            w = np.where(w > 0, w, 0.0)
            best = np.argsort(-w[begin:m - last], kind="stable")[:n - last - begin] + begin
            heads.append(sorted([*range(begin), *best.tolist(), *range(m - last, m)]))
        out.append(heads)
    return out


def evict_plan(lengths, keep, table, free, n_free, page):
    """One request and page after the other."""
    R, W = len(lengths), len(table[0])
    stack = [int(x) for x in free[:n_free]]
    out_len, out_table, back, asked, room = [], [], [], 0, len(stack)
    for r in range(R):
        have = min(-(-lengths[r] // page), W)
        row = [int(x) for x in table[r][:have]]
        if 0 <= keep[r] < lengths[r]:
            need = -(-keep[r] // page)
            asked += need
            if need == 0 or asked <= room:
                back += row
                row = [stack.pop() for _ in range(need)]
                out_len.append(int(keep[r]))
                out_table.append(row + [-1] * (W - len(row)))
                continue
        out_len.append(int(lengths[r]))
        out_table.append(row + [-1] * (W - len(row)))
    stack += back
    return dict(lengths=out_len, table=out_table, free=(stack + [-1] * len(free))[:len(free)], n_free=[min(len(stack), len(free))])
