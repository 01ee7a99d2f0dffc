"""Plain statements of the serving operators, in 64 bits on the CPU (codes and scales of the cache: in the 32 and 16 bits that its
format is defined in).  Written from the definitions in include/hyperattn.h."""
import math

import numpy as np
import torch

GROUP = 32


def quantise(x):
    """Codes, scales and minima of rows [..., d] by the format's definition."""
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], -1, GROUP)
    with np.errstate(all="ignore"):
        lo, hi = g.min(-1), g.max(-1)
        s = ((hi - lo) / np.float32(15)).astype(np.float16)
        m = lo.astype(np.float16)
        bad = ~np.isfinite(g).all(-1) | ~np.isfinite(s) | ~np.isfinite(m)
        s, m = np.where(bad, np.float16(np.nan), s), np.where(bad, np.float16(np.nan), m)
        r = np.where(s == 0, np.float32(0), np.float32(1) / s.astype(np.float32))
        c = np.rint((g - m.astype(np.float32)[..., None]) * r[..., None])
        codes = np.where(bad[..., None], 0, np.clip(c, 0, 15)).astype(np.uint8)
    return codes, s, m


def held(x):
    """The fp32 numbers that the cache holds in the place of rows [..., d]."""
    codes, s, m = quantise(x)
    return (m.astype(np.float32)[..., None] + s.astype(np.float32)[..., None] * codes).reshape(x.shape)


def block_bytes(k, v):
    """The bytes of one cache block, from K and V [16, d]."""
    d = k.shape[1]
    out = np.zeros(20 * d, np.uint8)
    for which, x in ((0, k), (1, v)):
        codes, s, m = quantise(x)
        codes = codes.reshape(16, d)
        for t in range(16):
            for c in range(d):
                code = int(codes[t, c])
                if which == 0:
                    lane, w, e = t % 8 * 4 + c // 8 % 4, c // 32, c % 8
                    at = ((t // 8) * 512 + lane * 16 if d == 128 else lane * 16 + t // 8 * 8) + w * 4
                    nibble = e % 2 * 4 + e // 2
                    out[at + nibble // 2] |= code << (4 * (nibble % 2))
                else:
                    u = c // 16
                    at = 8 * d + (u // 4) * 512 + (c % 8 * 4 + t % 8 // 2) * 16 + u % 4 * 4 + t % 2 * 2 + t // 8
                    out[at] |= code << (4 if c % 16 >= 8 else 0)
            for w in range(d // 32):
                at = 16 * d + which * 2 * d + (t // 2 * (d // 32) + w) * 8 + t % 2 * 2
                out[at:at + 2] = np.frombuffer(s[t, w].tobytes(), np.uint8)
                out[at + 4:at + 6] = np.frombuffer(m[t, w].tobytes(), np.uint8)
    return out


def plan(lengths, new, table, free, n_free, page, rows):
    """The scheduling step, one request and page after the other."""
    R, W = len(lengths), len(table[0])
    stack = [int(x) for x in free[:n_free]]
    out_table = [[-1] * W for _ in range(R)]
    out_len = [0] * R
    have = [-(-n // page) for n in lengths]
    for r in range(R):
        if new[r] < 0:
            stack += [int(x) for x in table[r][:have[r]]]
    room, asked, admitted = len(stack), 0, [False] * R
    for r in range(R):
        if new[r] < 0:
            continue
        out_len[r] = int(lengths[r])
        out_table[r][:have[r]] = [int(x) for x in table[r][:have[r]]]
        pages = -(-(lengths[r] + new[r]) // page)
        if pages > W:
            continue
        need = pages - have[r]
        asked += need
        if need == 0 or asked <= room:
            admitted[r] = True
            for c in range(have[r], pages):
                out_table[r][c] = stack.pop()
            out_len[r] += int(new[r])
    slots, positions, cu = [], [], [0]
    for r in range(R):
        for i in range(max(int(new[r]), 0)):
            pos = int(lengths[r]) + i
            page_id = out_table[r][pos // page] if admitted[r] else -1
            slots.append(page_id * page + pos % page if page_id >= 0 else -1)
            positions.append(pos if admitted[r] else -1)
        cu.append(cu[-1] + max(int(new[r]), 0))

    def cut(x):
        return (x + [-1] * rows)[:rows]

    return dict(slots=cut(slots), positions=cut(positions), cu_new=cu, cu_len=[0] + list(np.cumsum(out_len)), lengths=out_len, table=out_table,
                free=stack + [-1] * (len(free) - len(stack)), n_free=[len(stack)])


def attention(q, k, v, seen, scale=None):
    """q [n, d], k, v [m, d] (float64), row i sees the first seen[i] keys.  Returns out, lse, sum p |v| and the largest scale sum |q k|
    (what rounding errors of weights, values and scores are measured in)."""
    n, d = q.shape
    scale = scale or 1 / math.sqrt(d)
    out, lse, mass, size = np.zeros((n, d)), np.full(n, -np.inf), np.zeros((n, d)), np.zeros(n)
    with np.errstate(all="ignore"):
        for i in range(n):
            c = int(seen[i])
            if c <= 0:
                continue
            z = scale * (k[:c] @ q[i])
            top = z.max()
            e = np.exp(z - top) if top > -np.inf else np.zeros(c)
            total = e.sum()
            if total == 0:
                continue
            out[i], lse[i] = (e @ v[:c]) / total, top + np.log(total)
            mass[i], size[i] = (e @ np.abs(v[:c])) / total, scale * (np.abs(k[:c]) @ np.abs(q[i])).max()
    return out, lse, mass, size


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()
