"""The operators of the 4-bit key/value cache (page plan, write, read, attention) against their definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import kv4_ref as R

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def S():
    from paper_2605_17842_b200 import snlp
    return snlp


def cuda(a, dt=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dt is None else t.to(dt)).cuda()


def rounded(rng, shape, dtype, spread=1.0):
    """Random rows as the dtype holds them: (tensor on the GPU, the same values in float64)."""
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[-1:]) * 0.5)
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return t.cuda(), t.double().numpy()


# -- plan ----------------------------------------------------------------------------------------------------------------
def run_plan(S, ctx, new, page, max_tokens, width, free_extra=3, head=0, take=True, table=None):
    ctx, new = np.asarray(ctx, np.int32), np.asarray(new, np.int32)
    rng = np.random.default_rng(len(ctx) * 7 + page)
    B = len(ctx)
    have = [-(-int(max(c, 0)) // page) for c in ctx]
    total = sum(have) + sum(max(0, -(-(int(c) + int(n)) // page)) for c, n in zip(ctx, new) if int(c) + int(n) >= 0) + free_extra
    perm = rng.permutation(min(total, 10**6)).astype(np.int32)
    if table is None:
        table = np.full((B, width), -7, np.int32)
        at = 0
        for b, h in enumerate(have):
            m = min(h, width)
            table[b, :m] = perm[at:at + m]
            at += m
        free = perm[at:]
    else:
        free = perm
    want = R.plan(ctx, new, table, free if take else None, page, max_tokens, head)
    t = cuda(table)
    got = S.page_plan(cuda(ctx), cuda(new), t, page, max_tokens, free_pages=cuda(free) if take else None,
                      free_head=cuda(np.array([head], np.int32)) if head else None)
    for name, x, y in (("table", t, want[0]), ("slots", got.slots, want[1]), ("positions", got.positions, want[2]), ("cu", got.cu_new, want[3]),
                       ("lens", got.lens, want[4]), ("info", got.info, np.array(want[5:7]))):
        assert np.array_equal(x.cpu().numpy(), y), name
    return got, want


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("B", [1, 2, 33, 255, 256, 257, 700])
def test_plan_matches_a_loop(S, B, page):
    rng = np.random.default_rng(B + page)
    ctx, new = rng.integers(0, 300, B), rng.integers(0, 40, B)
    ctx[rng.random(B) < 0.2] = 0
    new[rng.random(B) < 0.2] = 0
    run_plan(S, ctx, new, page, int(new.sum()) + 9, 32, head=2)


def test_plan_edges(S):
    run_plan(S, [0], [0], 16, 0, 1)                    # nothing at all
    run_plan(S, [0, 0, 0], [0, 0, 0], 16, 4, 1)
    run_plan(S, [0], [1], 16, 1, 1)
    run_plan(S, [15, 16, 17], [1, 1, 1], 16, 3, 4)     # last of a page, first of the next, inside
    run_plan(S, [0], [5000], 64, 5000, 100)            # more tokens than one block serves
    run_plan(S, [31, 0], [1, 33], 32, 34, 2, free_extra=0)    # exactly enough pages


def test_plan_with_an_empty_free_list(S):
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    ctx, table = cuda(np.array([15, 4], np.int32)), cuda(np.array([[3, -1], [2, -1]], np.int32))
    served = S.page_plan(ctx, cuda(np.array([1, 5], np.int32)), table, 16, 6, free_pages=empty)      # no page is needed
    assert served.info.tolist() == [0, 0] and served.slots.tolist() == [63, 36, 37, 38, 39, 40]
    refused = S.page_plan(ctx, cuda(np.array([2, 5], np.int32)), table, 16, 7, free_pages=empty)
    assert refused.info.tolist() == [0, 1] and (refused.slots == -1).all() and (table[:, 1] == -1).all()


def test_bindings_refuse_what_they_cannot_pass_on(S):
    pool = S.kv4_pool(2, 2, 64, 16)
    k, sl = torch.zeros((3, 2, 64), dtype=BF, device="cuda"), torch.arange(3, device="cuda")
    q, t, n = torch.zeros((3, 2, 64), dtype=BF, device="cuda"), torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    for f in (lambda: S.kv4_write(pool, k[:2], k, sl), lambda: S.kv4_write(pool, k, k.float(), sl), lambda: S.kv4_write(pool, k.half(), k.half(), sl),
              lambda: S.kv4_write(pool, k, k, sl.int()), lambda: S.kv4_write(pool, k.transpose(1, 2).contiguous().transpose(1, 2), k, sl),
              lambda: S.kv4_write(pool.flatten(), k, k, sl), lambda: S.kv4_write(pool, k.cpu(), k, sl), lambda: S.kv4_read(pool, sl, 128),
              lambda: S.kv4_read(pool, sl, 64, torch.float16), lambda: S.kv4_pool(2, 2, 96, 16), lambda: S.kv4_pool(2, 2, 64, 24),
              lambda: S.kv4_attention(q[:, :, :32], pool, t, n), lambda: S.kv4_attention(q, pool, t, n[:2]), lambda: S.kv4_attention(q, pool, t.long(), n),
              lambda: S.kv4_attention(q, pool, t, n, cu_q=n), lambda: S.kv4_attention(q[:, :1].contiguous(), pool, t, n), lambda: S.kv4_attention(q, pool, t, n, out=q[:2]),
              lambda: S.kv4_attention(q, pool, t, n, max_len=-1), lambda: S.kv4_attention(q, pool, t, n, tile_rows=3), lambda: S.kv4_attention(q[:2], pool, t, n),
              lambda: S.page_plan(n, n, t[:2], 16, 3), lambda: S.page_plan(n, n.long(), t, 16, 3), lambda: S.page_plan(n, n, t, 16, -1), lambda: S.page_plan(n, n, t, 20, 3),
              lambda: S.page_plan(n, n, t, 16, 3, free_head=n), lambda: S.page_plan(n[:0], n[:0], t[:0], 16, 3)):
        with pytest.raises(S.SnlpError):
            f()
    assert torch.equal(S.kv4_attention(q[:0], pool, t, n, cu_q=torch.zeros(4, dtype=torch.int32, device="cuda")), q[:0])


def test_bindings_refuse_what_ctypes_would_cut(S):
    pool = S.kv4_pool(2, 2, 64, 16)
    q, t, n = torch.zeros((3, 2, 64), dtype=BF, device="cuda"), torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    sl, one = torch.arange(3, device="cuda"), torch.zeros((1, 2, 64), dtype=BF, device="cuda")
    for f in (lambda: S.kv4_attention(q, pool, t, n, max_len=(1 << 32) + 16), lambda: S.kv4_attention(q, pool, t, n, scale=0.0),
              lambda: S.kv4_attention(q, pool, t, n, scale=float("inf")), lambda: S.page_plan(n, n, t, 16, (1 << 32) + 3),
              lambda: S.kv4_read(pool, sl, 64, k=one.expand(3, 2, 64)), lambda: S.kv4_read(pool, sl, 64, k=q, v=q)):
        with pytest.raises(S.SnlpError):
            f()


def test_results_are_ordinary_tensors(S):
    """What the binding allocates can be changed in place, sliced, saved by autograd and freed in any order; pieces of one
    allocation do not reach into each other."""
    n, pool = torch.ones(3, dtype=torch.int32, device="cuda"), S.kv4_pool(3, 2, 64, 16)
    for mode in (torch.no_grad, torch.enable_grad, torch.inference_mode):
        with mode():
            table = torch.arange(3, dtype=torch.int32, device="cuda").reshape(3, 1)
            plan = S.page_plan(n * 0, n, table, 16, 4)
            assert [t.tolist() for t in plan] == [[0, 16, 32, -1], [0, 0, 0, -1], [0, 1, 2, 3], [1, 1, 1], [0, 0]]
            assert all(t.is_contiguous() and t.device == pool.device for t in plan)
            for i, t in enumerate(plan):
                before = [u.clone() for u in plan]
                t.add_(5)
                t[:1].zero_()
                assert t[0] == 0 and torch.equal(t[1:], before[i][1:] + 5)
                assert all(torch.equal(u, before[j]) for j, u in enumerate(plan) if j != i)
            keep = plan.lens.clone(), plan.lens
            del plan, t, before
            torch.empty(4096, dtype=torch.int32, device="cuda").fill_(9)
            assert torch.equal(*keep)
            k, v = S.kv4_read(pool.fill_(0), torch.arange(5, device="cuda"), 64)
            k.add_(1)
            assert (k == 1).all() and (v == 0).all()
            out = S.kv4_attention(k[:3], pool, table, n, max_len=16)
            assert (out.sub_(1) == -1).all()
    w = torch.ones(2, device="cuda", requires_grad=True)
    k, _ = S.kv4_read(pool.fill_(0), torch.arange(5, device="cuda"), 64, torch.float32)
    (w[0] * (k + 1)).sum().backward()
    assert w.grad.tolist() == [5 * 2 * 64, 0]


def test_bindings_name_what_is_not_a_tensor(S):
    pool, n = S.kv4_pool(3, 2, 64, 16), torch.ones(3, dtype=torch.int32, device="cuda")
    for f in (lambda: S.kv4_write(pool, None, None, n), lambda: S.kv4_read(pool, n.long(), 64, "bf16"), lambda: S.page_plan([1], n, n, 16, 3),
              lambda: S.kv4_attention(1.0, pool, n, n)):
        with pytest.raises(TypeError):
            f()


def test_plan_full_table_takes_nothing(S):
    table = np.arange(12, dtype=np.int32).reshape(3, 4)
    table[1, 2] = -1                                    # a hole: its tokens have no slot
    run_plan(S, [3, 30, 0], [20, 10, 1], 16, 40, 4, take=False, table=table)


@pytest.mark.parametrize("ctx,new,kw,bit", [
    ([40, 0], [8, 100], dict(width=8, free_extra=-5), 1),        # too few pages
    ([40, 0], [8, 100], dict(width=6), 2),                       # row too short
    ([40, 0], [8, 100], dict(width=8, max_tokens=107), 4),       # slot map too short
    ([40, -1], [8, 3], dict(width=8), 8),
    ([40, 1], [8, -3], dict(width=8), 8),
    ([2**31 - 1, 1], [1, 3], dict(width=8), 8),
])
def test_plan_refuses_whole(S, ctx, new, kw, bit):
    kw = dict(max_tokens=120, **kw) if "max_tokens" not in kw else kw
    got, want = run_plan(S, ctx, new, 16, kw.pop("max_tokens"), **kw)
    assert int(got.info[1]) & bit and int(got.info[0]) == 0
    assert (got.slots == -1).all()


# -- write and read --------------------------------------------------------------------------------------------------------
def check_rows(got, want, dtype):
    """got (tensor of dtype) is the rounding of want (fp32 sum s c + m of exact terms, then to dtype)."""
    g, w = got.double().cpu().numpy(), want
    assert np.array_equal(np.isnan(g), np.isnan(w))
    ok = ~np.isnan(w)
    # one rounding to fp32 (2^-24) and, for bf16, one more (2^-8); values at the bottom of the range: half a subnormal step
    rel = 2.0 ** -24 if dtype is F32 else 2.0 ** -8
    assert (np.abs(g - w)[ok] <= rel * 1.001 * np.abs(w[ok]) + 2.0 ** -133).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,heads,page", [(1, 1, 16), (5, 3, 16), (16, 2, 64), (17, 10, 64), (333, 7, 32), (1025, 1, 128)])
def test_write_read_round_trip(S, n, heads, page, dim, dtype):
    rng = np.random.default_rng(n * heads + dim)
    k, k64 = rounded(rng, (n, heads, dim), dtype)
    v, v64 = rounded(rng, (n, heads, dim), dtype)
    pages = -(-n // page) + 2
    slots = rng.permutation(pages * page)[:n]
    pool = S.kv4_pool(pages, heads, dim, page)
    pool.fill_(0xEE)
    S.kv4_write(pool, k, v, cuda(slots))
    for out in (BF, F32):
        gk, gv = S.kv4_read(pool, cuda(slots), dim, out)
        check_rows(gk, R.values(k64), out)
        check_rows(gv, R.values(v64), out)
    # the bytes themselves, where the format puts them, and nothing else was touched
    raw = pool.cpu().numpy()
    want = np.full_like(raw, 0xEE)
    cb, pb = 16 * dim // 2, 16 * dim // 16
    for i in range(min(n, 40) if n > 40 else n):
        pg, off = divmod(int(slots[i]), page)
        for h in range(heads):
            blk = want[pg, h, off // 16]
            t = off % 16
            for base, x, val in ((0, k64, False), (cb + pb, v64, True)):
                codes, par = R.pack_row(x[i, h], val)
                blk[base + t * dim // 2: base + (t + 1) * dim // 2] = np.frombuffer(codes, np.uint8)
                blk[base + cb + t * dim // 16: base + cb + (t + 1) * dim // 16] = np.frombuffer(par, np.uint8)
    if n <= 40:
        assert np.array_equal(raw, want)
    else:
        touched = want != 0xEE
        assert np.array_equal(raw[touched], want[touched])


def awkward(dim):
    """Rows at the borders of the format, float32 [rows, dim]."""
    rng = np.random.default_rng(1)
    one = np.ones(dim, np.float32)
    rows = [0 * one, one, -3.7 * one, one * 1e-38, one * 1e-45]
    r = rng.standard_normal(dim).astype(np.float32)
    rows += [r * f for f in (1e-40, 1e-36, 1e-30, 1e30, 2e38)]
    step = np.arange(dim, dtype=np.float32) % 16
    rows += [step, step + 0.5, np.where(step == 15, 15, np.minimum(step + 0.5, 14.5)).astype(np.float32)]   # ties
    t = step.copy(); t[3] = np.float32(6.5) + np.float32(2.0 ** -21); t[5] = np.float32(6.5) - np.float32(2.0 ** -21); rows.append(t)
    t = (step - 6.5).astype(np.float32); t[7] = 1e-30; t[9] = -1e-30; t[11] = 0; rows.append(t)     # the difference x - m is not exact
    for bad in (np.nan, np.inf, -np.inf):
        t = r.copy(); t[17] = bad; rows.append(t)
    t = r.copy(); t[0], t[1] = 3.4e38, -3.4e38; rows.append(t)      # the range itself overflows
    t = r.copy(); t[2] = -np.float32(3.4e38); rows.append(t)
    t = r * 1e-3 + np.float32(1000); rows.append(t.astype(np.float32))
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [64, 128])
def test_write_at_the_borders_of_the_format(S, dim, dtype):
    x = torch.from_numpy(awkward(dim)).to(dtype)
    n = len(x)
    pool = S.kv4_pool(4, 1, dim, 16)
    slots = torch.arange(n).cuda()
    S.kv4_write(pool, x[:, None].cuda(), x.flip(0)[:, None].contiguous().cuda(), slots)
    raw = pool.cpu().numpy()
    cb, pb = 16 * dim // 2, 16 * dim // 16
    x64 = x.double().numpy()
    for i in range(n):
        blk, t = raw[i // 16, 0, 0], i % 16
        for base, row, val in ((0, x64[i], False), (cb + pb, x64[n - 1 - i], True)):
            codes, par = R.pack_row(row, val)
            assert blk[base + cb + t * dim // 16: base + cb + (t + 1) * dim // 16].tobytes() == par, (i, val)
            assert blk[base + t * dim // 2: base + (t + 1) * dim // 2].tobytes() == codes, (i, val)
    k, v = S.kv4_read(pool, slots, dim, F32)
    check_rows(k[:, 0], R.values(x64), F32)


def test_write_fp32_codes_next_to_a_border(S):
    """Many fp32 values, a share of them moved next to the border of two codes: every code is the one of exact arithmetic."""
    rng = np.random.default_rng(5)
    n, dim = 4000, 64
    x = rng.standard_normal((n, 1, dim)).astype(np.float32)
    c, s, m = R.quantise(x.astype(np.float64))
    edge = (m + (np.clip(c, 0, 14) + 0.5).reshape(n, 1, 1, 64)[..., 0, :] * s).astype(np.float32)
    pick = rng.random(x.shape) < 0.3
    pick[..., :2] = False                      # leave some alone
    lohi = (x == x.min(-1, keepdims=True)) | (x == x.max(-1, keepdims=True))
    x = np.where(pick & ~lohi, np.nextafter(edge, np.where(rng.random(x.shape) < 0.5, np.float32(9), np.float32(-9))), x).astype(np.float32)
    pool = S.kv4_pool(n // 16, 1, dim, 16)
    slots = torch.arange(n).cuda()
    S.kv4_write(pool, cuda(x), cuda(x), slots)
    k, v = S.kv4_read(pool, slots, dim, F32)
    want = R.values(x.astype(np.float64))
    check_rows(k, want, F32)
    check_rows(v, want, F32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_write_takes_any_stride(S, dtype):
    """Keys and values as slices of a fused projection, at an odd offset, and broadcast over tokens."""
    rng = np.random.default_rng(3)
    n, heads, dim = 37, 3, 128
    big, b64 = rounded(rng, (n, 3 * heads * dim + 5), dtype, 0)
    slots = torch.arange(n).cuda()

    def go(k, v, k64, v64):
        pool = S.kv4_pool(3, heads, dim, 16)
        S.kv4_write(pool, k, v, slots)
        gk, gv = S.kv4_read(pool, slots, dim, F32)
        check_rows(gk, R.values(k64), F32)
        check_rows(gv, R.values(v64), F32)
    for off in (0, 1, 4, 5):
        cut = lambda x, i: x[:, off + i * heads * dim: off + (i + 1) * heads * dim].reshape(n, heads, dim) if isinstance(x, np.ndarray) \
            else x[:, off + i * heads * dim: off + (i + 1) * heads * dim].unflatten(1, (heads, dim))  # noqa: E731
        k, v = cut(big, 1), cut(big, 2)
        assert k.stride(0) == big.stride(0)
        go(k, v, cut(b64, 1), cut(b64, 2))
    one, o64 = rounded(rng, (1, heads, dim), dtype)
    go(one.expand(n, heads, dim), one.expand(n, heads, dim), np.broadcast_to(o64, (n, heads, dim)), np.broadcast_to(o64, (n, heads, dim)))
    tr, t64 = rounded(rng, (heads, n, dim), dtype)
    go(tr.transpose(0, 1), tr.transpose(0, 1), t64.swapaxes(0, 1), t64.swapaxes(0, 1))
    # read into strided rows: what lies between them stays
    pool = S.kv4_pool(3, heads, dim, 16)
    S.kv4_write(pool, tr.transpose(0, 1), tr.transpose(0, 1), slots)
    buf = torch.full((n, 2 * heads * dim + 3), 7.0, dtype=dtype, device="cuda")
    k, v = buf[:, 1:1 + heads * dim].unflatten(1, (heads, dim)), buf[:, 1 + heads * dim:1 + 2 * heads * dim].unflatten(1, (heads, dim))
    S.kv4_read(pool, slots, dim, dtype, k=k, v=v)
    check_rows(k, R.values(t64.swapaxes(0, 1)), dtype)
    assert (buf[:, 0] == 7).all() and (buf[:, -2:] == 7).all()


def test_slots_outside_the_pool(S):
    rng = np.random.default_rng(4)
    n, heads, dim, page = 20, 2, 64, 16
    k, k64 = rounded(rng, (n, heads, dim), BF)
    slots = np.arange(n)
    slots[[1, 7, 9, 19]] = [-1, 32, 2**40, -2**62]
    pool = S.kv4_pool(2, heads, dim, page)
    pool.fill_(0x11)
    before = pool.clone()
    S.kv4_write(pool, k, k, cuda(slots))
    gk, gv = S.kv4_read(pool, cuda(slots), dim, F32)
    want = R.values(k64)
    out = (slots < 0) | (slots >= 32)
    want[out] = 0
    check_rows(gk, want, F32)
    check_rows(gv, want, F32)
    untouched = [s for s in range(32) if s not in set(slots[~out])]
    assert untouched
    cb = 16 * dim // 2
    for s in untouched:
        pg, t = divmod(s, page)
        for base in (0, cb + 16 * dim // 16):
            assert torch.equal(pool[pg, :, 0, base + t * 32: base + (t + 1) * 32], before[pg, :, 0, base + t * 32: base + (t + 1) * 32])
    S.kv4_write(pool, k[:0], k[:0], cuda(slots[:0]))        # no token at all
    assert S.kv4_read(pool, cuda(slots[:0]), dim)[0].shape == (0, heads, dim)


# -- attention ---------------------------------------------------------------------------------------------------------------
class Cache:
    """A pool with sequences of given lengths on scattered pages; the rest of the pool is poisoned with NaN."""

    def __init__(self, S, lens, heads, dim, page, dtype=BF, seed=0, width=None, k_scale=1.0, v_scale=1.0):
        rng = np.random.default_rng(seed)
        self.S, self.lens, self.heads, self.dim, self.page = S, lens, heads, dim, page
        need = [max(0, -(-n // page)) for n in lens]
        self.pages = sum(need) + 3
        perm = rng.permutation(self.pages)
        self.table = np.full((len(lens), width or max(max(need), 1)), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = perm[at:at + m]
            at += m
        self.pool = S.kv4_pool(self.pages, heads, dim, page)
        self.pool.fill_(0xFF)                     # codes 15, parameters NaN
        self.k, self.v = [], []
        for b, n in enumerate(lens):
            n = max(n, 0)
            k, k64 = rounded(rng, (n, heads, dim), dtype)
            v, v64 = rounded(rng, (n, heads, dim), dtype)
            k, v = (k * k_scale).to(dtype), (v * v_scale).to(dtype)
            self.put(b, 0, k, v)
            self.k.append(R.values(k.double().cpu().numpy()) if n else np.zeros((0, heads, dim)))
            self.v.append(R.values(v.double().cpu().numpy()) if n else np.zeros((0, heads, dim)))

    def put(self, b, p0, k, v):
        p = np.arange(p0, p0 + len(k))
        self.S.kv4_write(self.pool, k, v, cuda(self.table[b, p // self.page].astype(np.int64) * self.page + p % self.page))

    def attend(self, q, cu=None, **kw):
        return self.S.kv4_attention(q, self.pool, cuda(self.table), cuda(np.array(self.lens, np.int32)), cu_q=cu, **kw)

    def check(self, out, q64, cu, dtype, scale=None, cut=None):
        scale = scale if scale is not None else 1 / math.sqrt(self.dim)
        got = out.double().cpu().numpy()
        for b, n in enumerate(self.lens):
            a, e = cu[b], cu[b + 1]
            if e == a:
                continue
            keys = min(max(n, 0), cut) if cut else max(n, 0)
            want, mag = R.attention(q64[a:e], self.k[b][:keys], self.v[b][:keys], n, scale)
            check_attention(got[a:e], want, mag, self.v[b][:keys], dtype)


def check_attention(got, want, mag, v, dtype):
    """Tolerance.  Scores: every product of a query term and a code is exact; the eight 16-term sums of a row, each with at most
    a unit (2^-23) of what has been added up, and the four roundings that apply the parameters stay below 2^-20 sum |q||k|
    (the terms s c and m of a key are of its size: |m| + s c <= 3 max|k|, so three of these); fp32 queries in two 11-bit terms
    add 2^-22.  A probability moves by twice the largest score error, and exp2 by 2^-21.  Second product: a warp adds at
    most 16 steps (2^-19).  bf16: probabilities to 11 bits (2^-11 of the value's distance from the group's low, which is at
    most the range of v) and the result to bf16 (2^-8)."""
    top = np.abs(v).max(initial=0.0)
    rel = 2 * (4 * 2.0 ** -20) * mag[..., None] + 2.0 ** -18
    tol = rel * top + np.zeros_like(want)
    if dtype is BF:
        tol += 2.0 ** -11 * (v.max(initial=0.0) - v.min(initial=0.0)) + 2.0 ** -8 * np.abs(want)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan)
    assert (np.abs(got - want)[~nan] <= tol[~nan]).all(), float((np.abs(got - want) / tol)[~nan].max())


def run_attention(S, lens, T, hq, hk, dim, page, dtype, seed=0, ragged=False, **kw):
    c = Cache(S, lens, hk, dim, page, dtype, seed, **kw)
    cu = np.concatenate([[0], np.cumsum(T if ragged else [T] * len(lens))])
    q, q64 = rounded(np.random.default_rng(seed + 99), (int(cu[-1]), hq, dim), dtype)
    out = c.attend(q, cuda(cu.astype(np.int32)) if ragged else None)
    c.check(out, q64, cu, dtype)
    return c, q, q64, out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 511, 1030])
def test_attention_single_token_lengths(S, n, dim, dtype):
    run_attention(S, [n], 1, 2, 2, dim, 16, dtype, seed=n)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 32, 64, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (10, 10), (4, 2), (6, 2), (8, 2), (7, 1), (24, 3), (9, 1)])
def test_attention_heads_and_pages(S, hq, hk, page, dtype):
    run_attention(S, [300, 7, 64, 129], 1, hq, hk, 128, page, dtype, seed=page + hq)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("T", [2, 3, 4, 7, 8, 9, 16, 17, 40])
def test_attention_blocks_of_rows(S, T, dim, dtype):
    run_attention(S, [T, T + 1, 270, 530], T, 4, 2, dim, 32, dtype, seed=T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_ragged_rows_and_empty_sequences(S, dtype):
    lens = [0, 300, 5, 0, 77, 1, 600, 40]
    rows = [0, 3, 5, 0, 1, 0, 33, 40]
    run_attention(S, lens, rows, 6, 3, 128, 16, dtype, ragged=True)


def test_attention_rows_without_keys_are_zero(S):
    # more rows than keys: the first rows stand before position 0; a sequence without keys
    c, q, q64, out = run_attention(S, [3, 0, 20], 8, 2, 2, 64, 16, BF)
    assert (out[:5] == 0).all() and (out[8:16] == 0).all() and (out[5:8] != 0).any()
    run_attention(S, [-5, 40], 1, 2, 2, 64, 16, F32)


def test_attention_rows_behind_the_last_sequence_stay(S):
    c = Cache(S, [50, 20], 2, 64, 16)
    q, q64 = rounded(np.random.default_rng(2), (9, 2, 64), BF)
    out = torch.full_like(q, 5.0)
    c.attend(q, cuda(np.array([0, 1, 4], np.int32)), out=out)
    assert (out[4:] == 5).all()
    c.check(out, q64, [0, 1, 4], BF)


@pytest.mark.parametrize("B,n,hk,G", [(2, 2500, 3, 1), (40, 700, 2, 3), (150, 1100, 2, 5)])     # every chunk length, more units than a batch
def test_attention_many_chunks(S, B, n, hk, G):
    rng = np.random.default_rng(B)
    lens = rng.integers(1, n + 1, B).tolist()
    lens[0] = n
    run_attention(S, lens, 1, hk * G, hk, 64, 64, F32)


@pytest.mark.parametrize("B,T,hk,G,n", [(1, 9, 2, 1, 900), (3, 40, 4, 4, 1500), (6, 40, 4, 4, 1500), (8, 40, 8, 4, 1100), (13, 40, 8, 4, 1100)])
def test_attention_every_split_of_prompt_chunks(S, B, T, hk, G, n):
    """Splits of 64, 128, 256, 512 and 1024 keys, by the number of row tiles."""
    run_attention(S, [n - 37 * b for b in range(B)], T, hk * G, hk, 64, 64, BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hk,n", [(1, 128), (1, 129), (3, 1030), (40, 2500), (160, 2100)])
def test_attention_every_split_of_single_tokens(S, hk, n, dtype):
    run_attention(S, [n, n // 2], 1, hk, hk, 64, 32, dtype)


def test_attention_of_thousands_of_sequences(S):
    """More sequences than the kernel's list has entries for, empty ones among them."""
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 40, 2500).tolist()
    run_attention(S, lens, rng.integers(0, 3, 2500).tolist(), 2, 1, 64, 16, F32, ragged=True)


def test_attention_long_splits(S):
    """A length bound beyond 256 splits of 512 keys: splits of 1024, more blocks than lanes."""
    c = Cache(S, [5000, 1030, 90], 1, 64, 16, F32, width=16385)
    q, q64 = rounded(np.random.default_rng(2), (3, 2, 64), F32)
    c.check(c.attend(q), q64, [0, 1, 2, 3], F32)
    two, q2, q264 = Cache(S, [4100], 2, 128, 64, BF, width=4097), *rounded(np.random.default_rng(3), (20, 2, 128), BF)
    two.check(two.attend(q2), q264, [0, 20], BF)


def test_attention_max_len_cuts_and_scale(S):
    c = Cache(S, [300, 90], 2, 128, 16)
    q, q64 = rounded(np.random.default_rng(2), (2, 2, 128), BF)
    c.check(c.attend(q, max_len=100), q64, [0, 1, 2], BF, cut=100)
    c.check(c.attend(q, max_len=4000, scale=0.31), q64, [0, 1, 2], BF, scale=0.31)
    wide = Cache(S, [300, 90], 2, 128, 16, width=700)        # a table far wider than the lengths
    wide.check(wide.attend(q), q64, [0, 1, 2], BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [-0.2, 1e-6, -0.03125])
def test_attention_takes_any_scale(S, scale, dtype):
    c = Cache(S, [300, 90, 17], 2, 64, 32, dtype)
    q, q64 = rounded(np.random.default_rng(3), (3, 4, 64), dtype)
    c.check(c.attend(q, scale=scale), q64, [0, 1, 2, 3], dtype, scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_scales_of_any_size(S, dtype):
    """Values and keys far from 1, and scales that grow and shrink along the sequence: the power of two that the
    probabilities are brought to has to follow."""
    for vs in (1e-20, 1e-6, 3e4, 1e20):
        run_attention(S, [300], 2, 2, 2, 64, 16, dtype, v_scale=vs)
    run_attention(S, [300], 2, 2, 2, 64, 16, dtype, k_scale=30.0)
    c = Cache(S, [500], 1, 128, 16, dtype)
    rng = np.random.default_rng(8)
    k, k64 = rounded(rng, (500, 1, 128), dtype)
    v, _ = rounded(rng, (500, 1, 128), dtype)
    v = (v * cuda(np.exp(4 * np.sin(np.arange(500) / 9.0)).astype(np.float32)).view(-1, 1, 1)).to(dtype)
    c.put(0, 0, k, v)
    c.k, c.v = [R.values(k64)], [R.values(v.double().cpu().numpy())]
    q, q64 = rounded(rng, (1, 4, 128), dtype)
    c.check(c.attend(q), q64, [0, 1], dtype)


def test_attention_query_of_any_size(S):
    c = Cache(S, [200], 2, 128, 16, F32)
    for f in (0.0, 1e-30, 1e-3, 50.0):
        q, q64 = rounded(np.random.default_rng(2), (3, 2, 128), F32)
        q, q64 = q * f, (q * f).double().cpu().numpy()
        c.check(c.attend(q), q64, [0, 3], F32)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_nan_reaches_only_who_sees_it(S, dtype):
    c = Cache(S, [200], 2, 128, 16, dtype)
    rng = np.random.default_rng(6)
    k, k64 = rounded(rng, (1, 2, 128), dtype)
    for which in ("k", "v"):
        c = Cache(S, [200], 2, 128, 16, dtype)
        x = k.clone()
        x[0, 1, 70] = float("inf")                 # head 1, second group, position 195
        c.put(0, 195, x if which == "k" else k, x if which == "v" else k)
        for store, val in ((c.k[0], x if which == "k" else k), (c.v[0], x if which == "v" else k)):
            store[195] = R.values(val.double().cpu().numpy())[0]
        q, q64 = rounded(rng, (8, 2, 128), dtype)   # rows at positions 192 .. 199
        out = c.attend(q)
        got = out.double().cpu().numpy()
        assert np.isfinite(got[:, 0]).all() and np.isfinite(got[:3]).all()
        if which == "k":
            assert np.isnan(got[3:, 1]).all()
        else:
            assert np.isnan(got[3:, 1, 64:]).all() and np.isfinite(got[3:, 1, :64]).all()
        want, mag = R.attention(q64[:3], c.k[0][:195], c.v[0][:195], 195, 1 / math.sqrt(128))
        check_attention(got[:3], want, mag, c.v[0][:195], dtype)
    c = Cache(S, [200], 2, 128, 16, dtype)
    for bad in (float("nan"), float("inf")):
        q, q64 = rounded(rng, (3, 2, 128), dtype)
        q[1, 0, 9] = bad
        got = c.attend(q).double().cpu().numpy()
        assert np.isnan(got[1, 0]).all() and np.isfinite(got[[0, 2]]).all() and np.isfinite(got[1, 1]).all()


@pytest.mark.parametrize("tile", [2, 4, 8, 16])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_row_does_not_depend_on_its_company(S, tile, dtype):
    """The same row bit for bit for one tile_rows: alone, within a block, with other lengths beside it; and right for each."""
    c = Cache(S, [700], 3, 128, 64, dtype)
    q, q64 = rounded(np.random.default_rng(2), (9, 3, 128), dtype)
    block = c.attend(q, tile_rows=tile)
    c.check(block, q64, [0, 9], dtype)
    for i in (0, 3, 8):
        one = Cache.__new__(Cache)
        one.__dict__.update(c.__dict__)
        one.lens = [700 - 8 + i]
        assert torch.equal(one.attend(q[i:i + 1].contiguous(), tile_rows=tile)[0], block[i])
    assert torch.equal(c.attend(q, tile_rows=tile), block)
    two, k, v = Cache(S, [700, 30], 3, 128, 64, dtype), *(rounded(np.random.default_rng(i), (700, 3, 128), dtype)[0] for i in (3, 4))
    c.put(0, 0, k, v)
    two.put(0, 0, k, v)
    assert torch.equal(two.attend(torch.cat([q[-1:], q[:1]]), tile_rows=tile)[0], c.attend(q[-1:].contiguous(), tile_rows=tile)[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_takes_any_query_stride(S, dtype):
    c = Cache(S, [100, 260], 2, 128, 16, dtype)
    rng = np.random.default_rng(2)
    big, b64 = rounded(rng, (6, 3 * 4 * 128 + 3), dtype, 0)
    for off in (0, 1, 8, 3):
        q = big[:, off:off + 4 * 128].unflatten(1, (4, 128))
        c.check(c.attend(q), b64[:, off:off + 4 * 128].reshape(6, 4, 128), [0, 3, 6], dtype)
    q = big[:, :4 * 128].unflatten(1, (4, 128)).transpose(0, 1).contiguous().transpose(0, 1)
    c.check(c.attend(q), b64[:, :4 * 128].reshape(6, 4, 128), [0, 3, 6], dtype)
    q = big[:1, :128].unflatten(1, (1, 128)).expand(6, 4, 128)
    c.check(c.attend(q), np.broadcast_to(b64[:1, :128].reshape(1, 1, 128), (6, 4, 128)), [0, 3, 6], dtype)


def test_attention_bad_pages_read_nothing(S):
    """Entries that are no page: their keys count as score 0 and value 0."""
    c = Cache(S, [200], 2, 64, 16, F32)
    c.table[0, [2, 5, 11]] = [-1, c.pages, 2**31 - 1]
    for j in (2, 5, 11):
        c.k[0][16 * j:16 * j + 16] = 0
        c.v[0][16 * j:16 * j + 16] = 0
    q, q64 = rounded(np.random.default_rng(2), (2, 2, 64), F32)
    c.check(c.attend(q), q64, [0, 2], F32)


def test_pool_beyond_32_bit_offsets(S):
    """The last page of a pool of more than 4 GB."""
    heads, dim, page = 16, 128, 64
    pages = (5 << 30) // (heads * page // 16 * 2304)
    c = Cache.__new__(Cache)
    c.S, c.lens, c.heads, c.dim, c.page, c.pages = S, [130], heads, dim, page, pages
    c.pool = S.kv4_pool(pages, heads, dim, page)
    assert c.pool.numel() > 1 << 32
    c.table = np.array([[pages - 1, pages - 2, pages // 2 + 1]], np.int32)
    rng = np.random.default_rng(1)
    k, k64 = rounded(rng, (130, heads, dim), BF)
    v, v64 = rounded(rng, (130, heads, dim), BF)
    c.put(0, 0, k, v)
    c.k, c.v = [R.values(k64)], [R.values(v64)]
    gk, gv = S.kv4_read(c.pool, cuda((c.table[0, np.arange(130) // page].astype(np.int64) * page + np.arange(130) % page)), dim, F32)
    check_rows(gk, c.k[0], F32)
    check_rows(gv, c.v[0], F32)
    q, q64 = rounded(rng, (2, heads, dim), BF)
    c.check(c.attend(q), q64, [0, 2], BF)


# -- together ------------------------------------------------------------------------------------------------------------------
def test_serving_loop(S):
    """Requests of different lengths through plan -> write -> attention, prompt chunks first, then single tokens, pages taken
    as they are needed; every step against attention in 64 bits over everything written so far."""
    rng = np.random.default_rng(11)
    B, hq, hk, dim, page = 4, 6, 3, 128, 16
    pages = 60
    pool = S.kv4_pool(pages, hk, dim, page)
    pool.fill_(0xFF)
    free = cuda(rng.permutation(pages).astype(np.int32))
    head = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.full((B, 16), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ks, vs = [np.zeros((0, hk, dim)) for _ in range(B)], [np.zeros((0, hk, dim)) for _ in range(B)]
    for new in ([5, 0, 40, 17], [1, 33, 1, 0], [1, 1, 1, 1], [1, 1, 1, 1], [15, 1, 0, 1], [1, 1, 1, 1]):
        n = sum(new)
        plan = S.page_plan(lens, cuda(np.array(new, np.int32)), table, page, n, free_pages=free, free_head=head)
        k, k64 = rounded(rng, (n, hk, dim), BF)
        v, v64 = rounded(rng, (n, hk, dim), BF)
        q, q64 = rounded(rng, (n, hq, dim), BF)
        S.kv4_write(pool, k, v, plan.slots)
        out = S.kv4_attention(q, pool, table, plan.lens, cu_q=plan.cu_new)
        assert plan.info.tolist()[1] == 0
        head, lens = head + plan.info[:1], plan.lens
        got, at = out.double().cpu().numpy(), 0
        for b in range(B):
            ks[b], vs[b] = np.concatenate([ks[b], R.values(k64[at:at + new[b]])]), np.concatenate([vs[b], R.values(v64[at:at + new[b]])])
            if new[b]:
                want, mag = R.attention(q64[at:at + new[b]], ks[b], vs[b], len(ks[b]), 1 / math.sqrt(dim))
                check_attention(got[at:at + new[b]], want, mag, vs[b], BF)
            at += new[b]
        assert lens.tolist() == [len(x) for x in ks]


def test_decode_step_in_a_graph_and_on_another_stream(S):
    """plan -> write -> attention captured once and replayed with other contents; then the same calls on a side stream."""
    rng = np.random.default_rng(12)
    B, h, dim, page = 3, 2, 64, 16
    c = Cache(S, [40, 17, 100], h, dim, page, width=10)
    used = set(c.table[c.table >= 0].tolist())
    free = cuda(np.array([p for p in range(c.pages) if p not in used], np.int32))
    table, ctx = cuda(c.table), cuda(np.array(c.lens, np.int32))
    new = torch.ones(B, dtype=torch.int32, device="cuda")
    k = torch.zeros((B, h, dim), dtype=BF, device="cuda")
    v, q = torch.zeros_like(k), torch.zeros_like(k)

    def step():
        plan = S.page_plan(ctx, new, table, page, B, free_pages=free)
        S.kv4_write(c.pool, k, v, plan.slots)
        return S.kv4_attention(q, c.pool, table, plan.lens), plan
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, plan = step()
    for rep in range(3):
        nk, k64 = rounded(rng, (B, h, dim), BF)
        nv, v64 = rounded(rng, (B, h, dim), BF)
        nq, q64 = rounded(rng, (B, h, dim), BF)
        k.copy_(nk); v.copy_(nv); q.copy_(nq)
        graph.replay()
        got = out.double().cpu().numpy()
        eager = step()[0]
        assert torch.equal(eager, out)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            other = step()[0]
        torch.cuda.synchronize()
        assert torch.equal(other, out)
        for b in range(B):
            n = c.lens[b]
            kk, vv = np.concatenate([c.k[b][:n], R.values(k64[b:b + 1])]), np.concatenate([c.v[b][:n], R.values(v64[b:b + 1])])
            want, mag = R.attention(q64[b:b + 1], kk, vv, n + 1, 1 / math.sqrt(dim))
            check_attention(got[b:b + 1], want, mag, vv, BF)
