"""Measured cases of the 4-bit key/value cache: page plan, write, read, attention.

Each case is one pass through an operator as a serving program calls it.  ``run`` computes it with elementary torch
operations where ``own`` is false and with this package's entry points where it is true; both work on the same pool of
pages, in the storage format of the library (``include/snlp.h``):

* pool: uint8 [page][kv head][page_size / 16][block]; a block holds 16 tokens of one head as
  key codes | key parameters | value codes | value parameters;
* a token's head_dim features are cut into groups of 64, each stored as 64 codes of 4 bits and a bf16 pair (scale, low):
  value = scale * code + low;
* eight consecutive features share a 32-bit word (feature i in bits 4i..4i+3); the words of a row are permuted
  (``_word_order``);
* slot = page * page_size + offset names a token's place, ``block_table[b][j]`` the page of positions
  j * page_size .. of sequence b.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64   # features that share a scale and a low
BLOCK = 16   # tokens of a storage block


# -- cases -----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # eight running requests, one new token each: the plan of a decode step
        {"name": "plan_decode_8", "op": "plan", "batch": 8, "ctx": 2048, "new": 1, "page": 64},
        # a queue of 400 ragged prompts, some of them continuations, planned at once
        {"name": "plan_prompts_400", "op": "plan", "batch": 400, "ctx": 1500, "new": 900, "page": 16},
        # the new keys and values of one decode step of one layer (10 heads of 128, batch 8), stored and read back
        {"name": "write_decode_8x10x128", "op": "write", "tokens": 8, "heads": 10, "dim": 128, "page": 64, "dtype": "bf16"},
        # a long prompt's keys and values of one layer, stored and read back
        {"name": "write_prompt_32768x8x128", "op": "write", "tokens": 32768, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # an odd number of tokens in fp32, small heads
        {"name": "write_fp32_5001x6x64", "op": "write", "tokens": 5001, "heads": 6, "dim": 64, "page": 32, "dtype": "fp32"},
        # one request's cache read back before its next prompt chunk is attended
        {"name": "read_2048x10x128", "op": "read", "tokens": 2048, "heads": 10, "dim": 128, "page": 64, "dtype": "bf16"},
        # eight requests' caches, small pages
        {"name": "read_70001x8x128", "op": "read", "tokens": 70001, "heads": 8, "dim": 128, "page": 16, "dtype": "bf16"},
        # single-token decoding: one request, 10 heads of 128, 2048 keys
        {"name": "attn_1x2048_h10", "op": "attn", "batch": 1, "len": 2048, "new": 1, "ragged": False, "q_heads": 10, "heads": 10, "dim": 128, "page": 64, "dtype": "bf16"},
        # the verify block of a draft: 9 rows over 4105 keys
        {"name": "attn_verify_9x4105_h10", "op": "attn", "batch": 1, "len": 4105, "new": 9, "ragged": False, "q_heads": 10, "heads": 10, "dim": 128, "page": 64, "dtype": "bf16"},
        # a large decode batch of ragged requests with grouped heads
        {"name": "attn_48x8192_h32_8", "op": "attn", "batch": 48, "len": 8192, "new": 1, "ragged": True, "q_heads": 32, "heads": 8, "dim": 128, "page": 64, "dtype": "bf16"},
        # fp32 inputs, heads of 64, ragged lengths, small pages
        {"name": "attn_fp32_7x1537_h12_6", "op": "attn", "batch": 7, "len": 1537, "new": 1, "ragged": True, "q_heads": 12, "heads": 6, "dim": 64, "page": 16, "dtype": "fp32"},
        # a mixed batch: prompt chunks of up to 200 rows beside continuations
        {"name": "attn_chunks_6x3000_h6", "op": "attn", "batch": 6, "len": 3000, "new": 200, "ragged": True, "q_heads": 6, "heads": 6, "dim": 128, "page": 32, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "write", "read", "attn", "attn", "attn"])
    page = rng.choice([16, 32, 64, 128])
    if op == "plan":
        return {"op": op, "batch": _log(rng, 1, 400), "ctx": _log(rng, 1, 1500), "new": _log(rng, 1, 900), "page": page}
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    dim = rng.choice([64, 128])
    heads = rng.randint(1, 10)
    if op in ("write", "read"):
        return {"op": op, "tokens": _log(rng, 1, 25000), "heads": heads, "dim": dim, "page": page, "dtype": dtype}
    group = rng.choice([1, 1, 2, 4, 7, 8])
    new = rng.choice([1, 1, 1, _log(rng, 2, 16), _log(rng, 17, 120)])
    batch = _log(rng, 1, 48 if new == 1 else 12)
    length = max(new, _log(rng, 1, 8192 if new == 1 else 3000))
    heads = min(heads, 8)
    if new > 16:
        heads = min(heads, 6)
        group = min(group, 2)
    return {"op": op, "batch": batch, "len": length, "new": new, "ragged": rng.random() < 0.6, "q_heads": heads * group, "heads": heads, "dim": dim,
            "page": page, "dtype": dtype}


# -- the storage format ------------------------------------------------------------------------------------------------
def _word_order(dim, value):
    """Position of the 32-bit word of features 8j..8j+7 within a row of codes."""
    ng = dim // GROUP
    j = np.arange(dim // 8)
    g, r = j // 8, j % 8
    return r * ng + g if value else (r // 2) * (2 * ng) + 2 * g + r % 2


def _quantise(x):
    """x [..., dim] -> codes uint8 [..., dim], scale and low bf16 [..., dim / 64]; in 64 bits: a value next to the border
    of two codes has to fall on its own side."""
    g = x.double().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    scale, low = ((hi - lo) / 15.0).float().bfloat16(), lo.float().bfloat16()
    bad = ~(torch.isfinite(scale) & torch.isfinite(low))
    s, m = scale.double()[..., None], low.double()[..., None]
    c = torch.where(s > 0, torch.round((g - m) / torch.where(s > 0, s, 1.0)), 0.0).clamp(0, 15)
    c = torch.where(bad[..., None], 0.0, c)
    nan = torch.full_like(scale, float("nan"))
    return c.flatten(-2).to(torch.uint8), torch.where(bad, nan, scale), torch.where(bad, nan, low)


def _rows(x, value):
    """x [n, heads, dim] -> (code bytes [n, heads, dim / 2], parameter bytes [n, heads, dim / 16])."""
    c, scale, low = _quantise(x)
    b = (c[..., 0::2] | (c[..., 1::2] << 4)).unflatten(-1, (-1, 4))
    order = torch.from_numpy(np.argsort(_word_order(x.shape[-1], value))).to(x.device)
    return b[..., order, :].flatten(-2), torch.stack([scale, low], -1).flatten(-2).contiguous().view(torch.uint8)


def _parts(dim):
    """Byte offsets of key codes, key parameters, value codes, value parameters within a block, and its size."""
    c, p = BLOCK * dim // 2, BLOCK * dim // 16
    return 0, c, c + p, 2 * c + p, 2 * (c + p)


def _store(pool, dim, page, slots, k, v):
    """Writes k, v [n, heads, dim] at slots [n] (elementary indexing)."""
    ok = (slots >= 0) & (slots < pool.shape[0] * page)
    slots, k, v = slots[ok], k[ok], v[ok]
    kc, kp, vc, vp, size = _parts(dim)
    flat = pool.view(pool.shape[0], pool.shape[1], page // BLOCK, size)
    pg, blk, tok = slots // page, (slots % page) // BLOCK, slots % BLOCK
    for base, half, x in ((0, 0, k), (vc, 1, v)):   # the two tensors, not the data
        codes, par = _rows(x, bool(half))
        n, h = codes.shape[:2]
        for at, b in ((base, codes), (base + kp, par)):
            w = b.shape[-1]
            part = flat[..., at:at + BLOCK * w].unflatten(-1, (BLOCK, w))
            part[pg[:, None], torch.arange(h, device=b.device)[None], blk[:, None], tok[:, None]] = b


def _unrow(codes, par, value):
    """(code bytes [..., dim / 2], parameter bytes [..., dim / 16]) -> values fp32 [..., dim]."""
    dim = codes.shape[-1] * 2
    order = torch.from_numpy(_word_order(dim, value)).to(codes.device)
    b = codes.unflatten(-1, (-1, 4))[..., order, :].flatten(-2)
    c = torch.stack([b & 15, b >> 4], -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    p = par.contiguous().view(torch.bfloat16).float().unflatten(-1, (-1, 2))
    return (p[..., 0:1] * c + p[..., 1:2]).flatten(-2)


def _load(pool, dim, page, slots):
    """Values k, v [n, heads, dim] fp32 at slots [n]."""
    kc, kp, vc, vp, size = _parts(dim)
    rows = pool.view(pool.shape[0], pool.shape[1], page // BLOCK, size)[slots // page, :, (slots % page) // BLOCK]
    tok, i = slots % BLOCK, torch.arange(len(slots), device=slots.device)

    def part(at, w):
        return rows[..., at:at + BLOCK * w].unflatten(-1, (BLOCK, w))[i, :, tok]
    return (_unrow(part(kc, dim // 2), part(kp, dim // 16), False), _unrow(part(vc, dim // 2), part(vp, dim // 16), True))


# -- inputs ------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, gen):
    """Total length and new rows of each sequence: the case says which lengths there are, `gen` in what order."""
    b, n, t = case["batch"], case["len"], case["new"]
    if not case["ragged"]:
        return np.full(b, n), np.full(b, t)
    own_gen = np.random.default_rng([b, n, t])
    t_b = own_gen.integers(1, t + 1, b)
    n_b = np.maximum(own_gen.integers(max(1, n // 8), n + 1, b), t_b)
    n_b[0], t_b[0] = n, t   # the longest is there
    order = gen.permutation(b)
    return n_b[order], t_b[order]


def _plan_lengths(case, gen):
    """Cached and new lengths of each sequence, likewise."""
    b = case["batch"]
    own_gen = np.random.default_rng([b, case["ctx"], case["new"]])
    ctx = own_gen.integers(0, case["ctx"] + 1, b)
    new = own_gen.integers(0, case["new"] + 1, b) if case["new"] > 1 else np.ones(b, np.int64)
    order = gen.permutation(b)
    return ctx[order].astype(np.int32), new[order].astype(np.int32)


def _shape(case, seed):
    """What of the inputs the host knows: lengths, tables, page count (numpy, from the seed)."""
    gen = np.random.default_rng(seed)
    if case["op"] == "attn":
        n_b, t_b = _lengths(case, gen)
        need = -(-n_b // case["page"])
        pages = int(need.sum())
        perm = gen.permutation(pages)
        table = np.full((case["batch"], int(need.max())), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = perm[at:at + m]
            at += m
        return n_b, t_b, table, pages
    pages = -(-case["tokens"] // case["page"]) + 3
    perm = gen.permutation(pages)
    i = np.arange(case["tokens"])
    return perm[i // case["page"]].astype(np.int64) * case["page"] + i % case["page"], pages


def _normal(gen, shape):
    """Keys after the per-head norm and values: unit scale, some features larger than others in every head."""
    x = torch.randn(shape, generator=gen, device="cuda")
    return x * (0.5 + torch.rand(shape[1:], generator=gen, device="cuda") * 1.5)


def prepare(case, seed):
    if case["op"] == "plan":
        rng = np.random.default_rng(seed)
        b, page = case["batch"], case["page"]
        ctx, new = _plan_lengths(case, rng)
        have = -(-ctx.astype(np.int64) // page)
        need = -(-(ctx.astype(np.int64) + new) // page)
        width = int(-(-(case["ctx"] + case["new"]) // page))
        perm = rng.permutation(int(need.sum()) + 7).astype(np.int32)
        table = np.full((b, width), -1, np.int32)
        at = 0
        for i, h in enumerate(have):
            table[i, :h] = perm[at:at + h]
            at += h
        cuda = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        return {"case": case, "ctx": cuda(ctx), "new": cuda(new), "table": cuda(table), "free": cuda(perm[at:]), "max_tokens": int(new.sum()) + 5}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dim, page, heads, dt = case["dim"], case["page"], case["heads"], _dtype(case)
    size = _parts(dim)[4]
    if case["op"] in ("write", "read"):
        slots, pages = _shape(case, seed)
        n = case["tokens"]
        k, v = _normal(gen, (n, heads, dim)).to(dt), _normal(gen, (n, heads, dim)).to(dt)
        pool = torch.zeros((pages, heads, page // BLOCK, size), dtype=torch.uint8, device="cuda")
        slots = torch.from_numpy(slots).cuda()
        if case["op"] == "write":
            return {"case": case, "pool": pool, "k": k, "v": v, "slots": slots}
        _store(pool, dim, page, slots, k, v)
        return {"case": case, "pool": pool, "slots": slots}
    n_b, t_b, table, pages = _shape(case, seed)
    pool = torch.zeros((pages, heads, page // BLOCK, size), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 14) // page)
    for p0 in range(0, pages, step):   # pages are filled in runs, whatever sequence they belong to
        n = (min(pages, p0 + step) - p0) * page
        slots = torch.arange(p0 * page, p0 * page + n, device="cuda")
        _store(pool, dim, page, slots, _normal(gen, (n, heads, dim)), _normal(gen, (n, heads, dim)))
    total = int(t_b.sum())
    q = (_normal(gen, (total, case["q_heads"], dim))).to(dt)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
    cu = np.concatenate([[0], np.cumsum(t_b)])
    return {"case": case, "pool": pool, "q": q, "table": i32(table), "lens": i32(n_b), "cu": i32(cu), "uniform": bool((t_b == t_b[0]).all()),
            "t_max": int(t_b.max()), "n_max": int(n_b.max())}


# -- one pass ----------------------------------------------------------------------------------------------------------
def _plain_plan(s):
    page, ctx, new, table, free = s["case"]["page"], s["ctx"].long(), s["new"].long(), s["table"], s["free"]
    have, need = (ctx + page - 1) // page, (ctx + new + page - 1) // page
    cu = torch.cat([torch.zeros_like(ctx[:1]), new.cumsum(0)])
    off = (need - have).cumsum(0) - (need - have)
    j = torch.arange(table.shape[1], device=table.device)[None]
    fresh = (j >= have[:, None]) & (j < need[:, None])
    pick = (off[:, None] + j - have[:, None]).clamp(0, len(free) - 1)
    table.copy_(torch.where(fresh, free[pick], table))
    i = torch.arange(s["max_tokens"], device=table.device)
    live = i < cu[-1]
    b = (torch.searchsorted(cu, i, right=True) - 1).clamp(0, len(ctx) - 1)
    pos = torch.where(live, ctx[b] + i - cu[b], 0)
    slots = torch.where(live, table[b, pos // page].long() * page + pos % page, -1)
    return {"table": table, "slots": slots, "positions": torch.where(live, pos, -1).int(), "cu": cu.int(), "lens": (ctx + new).int(),
            "used": (need - have).sum().int()}


def _plain_attention(s):
    c, pool, table = s["case"], s["pool"], s["table"].long()
    page, dim, hk, hq = c["page"], c["dim"], c["heads"], c["q_heads"]
    lens, cu = s["lens"].long(), s["cu"].long()
    t_b = cu[1:] - cu[:-1]
    b, width = table.shape
    kc, kp, vc, vp, size = _parts(dim)
    raw = pool[table.clamp(min=0)]                                               # [b, width, heads, page / 16, block]

    def part(at, w):
        x = raw[..., at:at + BLOCK * w].unflatten(-1, (BLOCK, w)).transpose(2, 3)  # [b, width, page / 16, heads, 16, w]
        return x.transpose(3, 4).reshape(b, width * page, hk, w).transpose(1, 2)
    k = _unrow(part(kc, dim // 2), part(kp, dim // 16), False)                   # [b, heads, n, dim]
    v = _unrow(part(vc, dim // 2), part(vp, dim // 16), True)
    i = torch.arange(s["t_max"], device=table.device)
    live = i[None] < t_b[:, None]
    row = torch.where(live, cu[:-1, None] + i[None], 0)                          # [b, t]
    q = s["q"].float()[row].unflatten(2, (hk, hq // hk))                          # [b, t, heads, group, dim]
    w = torch.einsum("bthgd,bhnd->bhgtn", q, k) / math.sqrt(dim)
    key = torch.arange(width * page, device=table.device)
    seen = key[None, None] <= (lens - t_b)[:, None, None] + i[None, :, None]      # [b, t, n]
    w = w.masked_fill(~seen[:, None, None], float("-inf"))
    w = torch.exp(w - w.amax(-1, keepdim=True))
    v = torch.where((key[None] < lens[:, None])[:, None, :, None], v, 0.0)
    o = torch.einsum("bhgtn,bhnd->bthgd", w, v) / w.sum(-1).permute(0, 3, 1, 2)[..., None]
    tok = torch.arange(len(s["q"]), device=table.device)
    tb = torch.searchsorted(cu, tok, right=True) - 1
    return o.flatten(2, 3)[tb, tok - cu[tb]].to(s["q"].dtype)


def run(state):
    c = state["case"]
    op = c["op"]
    if own:
        from paper_2605_17842_b200 import snlp
        if op == "plan":
            p = snlp.page_plan(state["ctx"], state["new"], state["table"], c["page"], state["max_tokens"], free_pages=state["free"])
            return {"table": state["table"], "slots": p.slots, "positions": p.positions, "cu": p.cu_new, "lens": p.lens, "used": p.info[0]}
        if op == "write":
            snlp.kv4_write(state["pool"], state["k"], state["v"], state["slots"])
            k, v = snlp.kv4_read(state["pool"], state["slots"], c["dim"], state["k"].dtype)
            return {"k": k, "v": v}
        if op == "read":
            k, v = snlp.kv4_read(state["pool"], state["slots"], c["dim"], _dtype(c))
            return {"k": k, "v": v}
        return snlp.kv4_attention(state["q"], state["pool"], state["table"], state["lens"], cu_q=None if state["uniform"] else state["cu"],
                                  max_len=state["n_max"])
    if op == "plan":
        return _plain_plan(state)
    if op == "write":
        _store(state["pool"], c["dim"], c["page"], state["slots"], state["k"], state["v"])
    if op in ("write", "read"):
        k, v = _load(state["pool"], c["dim"], c["page"], state["slots"])
        return {"k": k.to(_dtype(c)), "v": v.to(_dtype(c))}
    return _plain_attention(state)


# -- what a pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    if case["op"] == "plan":
        ctx, new = _plan_lengths(case, np.random.default_rng(0))
        b, n, page = case["batch"], int(new.sum()) + 5, case["page"]
        fresh = int((-(-(ctx + new) // page) + (-ctx // page)).sum())   # page numbers taken from the free list into the table
        return {"bytes": b * 16 + n * 12 + fresh * 8 + 4, "flops": b * 6 + n * 4}
    dim, heads, esz = case["dim"], case["heads"], 2 if case["dtype"] == "bf16" else 4
    held = 2 * (dim // 2 + dim // 16)                      # bytes of one token of one head
    if case["op"] in ("write", "read"):
        n = case["tokens"] * heads
        full = 2 * dim * esz
        passes = 2 if case["op"] == "write" else 1         # stored, and read back
        return {"bytes": passes * n * (held + full) + passes * 8 * case["tokens"], "flops": passes * n * dim * 4}
    n_b, t_b, table, pages = _shape(case, 0)
    seen = sum(int(t) * int(n) - int(t) * (int(t) - 1) // 2 for n, t in zip(n_b, t_b))
    return {"bytes": int(n_b.sum()) * heads * held + 2 * int(t_b.sum()) * case["q_heads"] * dim * esz + 4 * table.size,
            "flops": 4 * seen * case["q_heads"] * dim}


# -- the definition in 64 bits -------------------------------------------------------------------------------------------
def _exact_plan(s):
    page, ctx, new = s["case"]["page"], s["ctx"].tolist(), s["new"].tolist()
    table, free = s["table"].cpu().numpy().copy(), s["free"].tolist()
    slots, pos, cu, used = [], [], [0], 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        for j in range((c + page - 1) // page, (c + n + page - 1) // page):
            table[b, j] = free[used]
            used += 1
        p = np.arange(c, c + n, dtype=np.int64)
        slots.append(table[b, p // page].astype(np.int64) * page + p % page)
        pos.append(p)
        cu.append(cu[-1] + n)
    rest = np.full(s["max_tokens"] - cu[-1], -1, np.int64)
    return {"table": torch.from_numpy(table), "slots": torch.from_numpy(np.concatenate(slots + [rest])),
            "positions": torch.from_numpy(np.concatenate(pos + [rest]).astype(np.int32)), "cu": torch.tensor(cu, dtype=torch.int32),
            "lens": torch.tensor([c + n for c, n in zip(ctx, new)], dtype=torch.int32), "used": torch.tensor(used, dtype=torch.int32)}


def _exact_group(x):
    """The value a 4-bit group stands for, x [..., 64] in float64."""
    lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    s, m = ((hi - lo) / 15).float().to(torch.bfloat16).double(), lo.float().to(torch.bfloat16).double()
    c = torch.clamp(torch.round((x - m) / s.clamp(min=1e-300)), 0, 15)
    return torch.where(s > 0, s * c + m, m)


def _exact_rows(raw, dim, value):
    """Values in float64 of the 16 rows of every block, raw: uint8 [..., block] -> [..., 16, dim]."""
    at = (BLOCK * (dim // 2 + dim // 16)) if value else 0
    ng = dim // GROUP
    out = torch.empty(raw.shape[:-1] + (BLOCK, dim), dtype=torch.float64, device=raw.device)
    words = raw[..., at:at + BLOCK * dim // 2].reshape(raw.shape[:-1] + (BLOCK, dim // 2))
    par = raw[..., at + BLOCK * dim // 2:at + BLOCK * (dim // 2 + dim // 16)].reshape(raw.shape[:-1] + (BLOCK, ng, 2, 2)).int()
    num = (((par[..., 1] << 8) | par[..., 0]) << 16).view(torch.float32).double()          # bf16 bits -> value
    for f in range(dim):
        g, r = f // GROUP, (f % GROUP) // 8
        word = r * ng + g if value else (r // 2) * 2 * ng + 2 * g + r % 2
        byte = words[..., 4 * word + (f % 8) // 2]
        code = (byte >> 4 if f % 2 else byte & 15).double()
        out[..., f] = num[..., g, 0] * code + num[..., g, 1]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "plan":
        return _exact_plan(s)
    dim, page = case["dim"], case["page"]
    if op == "write":
        return {n: _exact_group(s[n].double().unflatten(-1, (-1, GROUP))).flatten(-2) for n in ("k", "v")}
    if op == "read":
        found = {"k": [], "v": []}
        for at in s["slots"].split(4096):
            raw = s["pool"][at // page, :, (at % page) // BLOCK]
            i = torch.arange(len(at), device=at.device)
            for n in found:
                found[n].append(_exact_rows(raw, dim, n == "v")[i, :, at % BLOCK])
        return {n: torch.cat(x) for n, x in found.items()}
    hk, group, out = case["heads"], case["q_heads"] // case["heads"], []
    for b, n in enumerate(s["lens"].tolist()):
        a, e = s["cu"][b].item(), s["cu"][b + 1].item()
        raw = s["pool"][s["table"][b, :-(-n // page)].long()].transpose(0, 1)               # [heads, pages, page / 16, block]
        k, v = (_exact_rows(raw, dim, w).reshape(hk, -1, dim)[:, :n] for w in (False, True))
        q = s["q"][a:e].double().reshape(e - a, hk, group, dim).permute(1, 2, 0, 3)          # [heads, group, t, dim]
        w = q @ k[:, None].transpose(-1, -2) / math.sqrt(dim)
        hide = torch.arange(n, device=q.device)[None] > n - (e - a) + torch.arange(e - a, device=q.device)[:, None]
        o = torch.softmax(w.masked_fill(hide, float("-inf")), -1) @ v[:, None]
        out.append(o.permute(2, 0, 1, 3).reshape(e - a, hk * group, dim))
    return torch.cat(out)
