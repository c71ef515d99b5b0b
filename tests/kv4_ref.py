"""The 4-bit key/value cache written out in numpy and 64 bits, from its definition in include/snlp.h."""
from fractions import Fraction

import numpy as np


def bf16(x):
    """float32 array -> nearest bf16 (ties to even), as float64; NaN and overflow to infinity as the format has them."""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.nan, r).astype(np.float64)


def quantise(x):
    """x [..., dim] -> codes [..., dim] int, scale, low [..., dim / 64] float64."""
    with np.errstate(all="ignore"):
        g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (x.shape[-1] // 64, 64))
        lo, hi = g.min(-1), g.max(-1)
        s, m = bf16(((hi - lo) / 15.0).astype(np.float32)), bf16(lo.astype(np.float32))
        bad = ~(np.isfinite(s) & np.isfinite(m))
        s, m = np.where(bad, np.nan, s), np.where(bad, np.nan, m)
        q = (g - m[..., None]) / s[..., None]
        r = np.rint(q)
        # next to the border of two codes 64 bits may round the difference itself (1e-30 + 6.5 is 6.5 there): exact fractions
        for at in zip(*np.nonzero((s[..., None] > 0) & (np.abs(q - np.floor(q) - 0.5) < 1e-9) & (np.abs(q) < 100))):
            r[at] = round((Fraction(g[at]) - Fraction(m[at[:-1]])) / Fraction(s[at[:-1]]))     # ties to even
        c = np.where(s[..., None] > 0, np.clip(r, 0, 15), 0.0)
    return c.reshape(x.shape).astype(np.int64), s, m


def values(x):
    """What a row stands for once stored: [..., dim] float64."""
    c, s, m = quantise(x)
    g = c.reshape(x.shape[:-1] + (x.shape[-1] // 64, 64))
    return (s[..., None] * g + m[..., None]).reshape(x.shape)


def word_place(dim, value):
    n = dim // 64
    return [((j % 8) * n + j // 8) if value else ((j % 8) // 2) * 2 * n + 2 * (j // 8) + j % 2 for j in range(dim // 8)]


def pack_row(x, value):
    """Bytes of codes and of parameters of one row x [dim]."""
    c, s, m = quantise(x)
    dim = x.shape[-1]
    words = [0] * (dim // 8)
    for j, at in enumerate(word_place(dim, value)):
        words[at] = sum(int(c[8 * j + i]) << (4 * i) for i in range(8))
    par = np.empty((dim // 64, 2), np.float32)
    par[:, 0], par[:, 1] = s, m
    bits = (par.view(np.uint32) >> 16).astype(np.uint16)
    bits = np.where(np.isnan(par), 0x7FC0, bits).astype("<u2")
    return np.array(words, "<u4").tobytes(), bits.tobytes()


def plan(ctx, new, table, free, page, max_tokens, head=0):
    """(table, slots, positions, cu, lens, used, status) by a loop over the tokens."""
    table, B, width = table.copy(), len(ctx), table.shape[1]
    ctx, new = [int(c) for c in ctx], [int(n) for n in new]
    status = 0
    if any(c < 0 or n < 0 or c + n > 2**31 - 1 for c, n in zip(ctx, new)):
        status |= 8
    ok = [c >= 0 and n >= 0 and c + n <= 2**31 - 1 for c, n in zip(ctx, new)]
    need = sum(-(-(c + n) // page) - -(-c // page) for c, n, k in zip(ctx, new, ok) if k)
    if any(-(-(c + n) // page) > width for c, n, k in zip(ctx, new, ok) if k):
        status |= 2
    if free is not None and need > 0 and need > len(free) - head:
        status |= 1
    if sum(n for n, k in zip(new, ok) if k) > max_tokens:
        status |= 4
    slots, pos = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int32)
    if status:
        return table, slots, pos, np.zeros(B + 1, np.int32), np.maximum(ctx, 0).astype(np.int32), 0, status
    at, i, cu = head, 0, [0]
    for b in range(B):
        for p in range(int(ctx[b]), int(ctx[b] + new[b])):
            if p % page == 0 and free is not None:
                table[b, p // page] = free[at]
                at += 1
            e = int(table[b, p // page])
            slots[i], pos[i] = (e * page + p % page if e >= 0 else -1), p
            i += 1
        cu.append(i)
    return table, slots, pos, np.array(cu, np.int32), (np.asarray(ctx) + np.asarray(new)).astype(np.int32), at - head, 0


def attention(q, k, v, length, scale):
    """One sequence: q [T, Hq, dim], k, v [n, Hkv, dim] (n = keys that are there, length = the sequence's length) -> (out,
    bound of the score error per row in units of 2^-20) in float64."""
    T, Hq, dim = q.shape
    n, Hkv = k.shape[:2]
    out, mag = np.zeros(q.shape), np.zeros((T, Hq))
    for h in range(Hq):
        kk, vv = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
        for i in range(T):
            vis = min(max(length - T + i + 1, 0), n)
            if vis == 0:
                continue
            with np.errstate(all="ignore"):
                s = (kk[:vis] @ q[i, h]) * scale
                w = np.exp(s - s.max())
                out[i, h] = (w @ vv[:vis]) / w.sum()
                mag[i, h] = abs(scale) * (np.abs(kk[:vis]) @ np.abs(q[i, h])).max()
    return out, mag
