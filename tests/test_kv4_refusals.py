"""What the entry points of the 4-bit cache refuse: every call here is turned away on the host, before any launch."""
import ctypes as C

import pytest

from paper_2605_17842_b200 import build

build.build()
from paper_2605_17842_b200 import snlp  # noqa: E402

lib = snlp.raw_library()
P = 1 << 20          # a well-aligned address that nothing may look at


def pool(pages=P, n_pages=4, page=16, heads=2, dim=64):
    return snlp.Kv4Pool(pages, n_pages, page, heads, dim)


def attn(**kw):
    d = dict(q=P, q_token_stride=256, q_head_stride=64, block_table=P, lens=P, cu_q=None, dtype=1, n_rows=2, B=2, n_head=4, max_pages=8, max_len=0, tile_rows=0, scale=0.0)
    d.update(kw)
    return snlp.Kv4Attn(*[d[n] for n, _ in snlp.Kv4Attn._fields_])


def message():
    return lib.snlp_last_error().decode()


@pytest.mark.parametrize("p,code", [
    (pool(page=8), snlp.ERR_ARG), (pool(page=48), snlp.ERR_ARG), (pool(page=2048), snlp.ERR_ARG), (pool(n_pages=0), snlp.ERR_ARG), (pool(heads=0), snlp.ERR_ARG),
    (pool(dim=32), snlp.ERR_UNSUPPORTED), (pool(dim=96), snlp.ERR_UNSUPPORTED), (pool(dim=256), snlp.ERR_UNSUPPORTED),
])
def test_pool_geometry(p, code):
    n = C.c_size_t()
    assert lib.snlp_kv4_pool_bytes(C.byref(p), C.byref(n)) == code and "snlp_kv4_pool_bytes" in message()
    assert lib.snlp_kv4_write(C.byref(p), C.c_void_p(P), C.c_void_p(P), 1, None, C.c_void_p(P), 1, None) == code
    assert lib.snlp_kv4_read(C.byref(p), C.c_void_p(P), C.c_void_p(P), 1, None, C.c_void_p(P), 1, None) == code
    assert lib.snlp_kv4_attention(C.byref(p), C.byref(attn()), C.c_void_p(P), None, C.c_size_t(0), None) == code


def test_pool_bytes():
    n = C.c_size_t()
    for dim, block in ((64, 1152), (128, 2304)):
        assert lib.snlp_kv4_pool_bytes(C.byref(pool(pages=None, n_pages=100000, page=64, heads=16, dim=dim)), C.byref(n)) == 0
        assert n.value == 100000 * 16 * 4 * block       # beyond 32 bits
    assert lib.snlp_kv4_pool_bytes(None, C.byref(n)) == snlp.ERR_ARG
    assert lib.snlp_kv4_pool_bytes(C.byref(pool()), None) == snlp.ERR_ARG


@pytest.mark.parametrize("fn", ["snlp_kv4_write", "snlp_kv4_read"])
def test_rows(fn):
    f = getattr(lib, fn)
    p = C.byref(pool())
    go = lambda pl=p, k=P, v=P, dt=1, st=None, s=P, n=1: f(pl, C.c_void_p(k), C.c_void_p(v), dt, st, C.c_void_p(s), n, None)  # noqa: E731
    for bad in (dict(pl=None), dict(k=0), dict(v=0), dict(s=0), dict(dt=2), dict(dt=-1), dict(n=-1), dict(k=P + 1), dict(s=P + 4), dict(v=P + 2, dt=0),
                dict(st=(C.c_int64 * 4)(-1, 1, 1, 1)), dict(pl=C.byref(pool(pages=P + 8))), dict(pl=C.byref(pool(pages=None)))):
        assert go(**bad) == snlp.ERR_ARG, bad
        assert fn in message()
    assert go(n=0) == 0 and go(n=0, k=0, v=0, s=0) == 0      # no token: nothing to do


def test_plan():
    def go(ctx=P, new=2 * P, B=2, page=16, free=P, nf=4, head=0, table=P, width=4, most=8, slots=P, pos=P, cu=P, lens=3 * P, info=P):
        v = C.c_void_p
        return lib.snlp_page_plan(v(ctx), v(new), B, page, v(free), nf, v(head), v(table), width, most, v(slots), v(pos), v(cu), v(lens), v(info), None)
    for bad in (dict(ctx=0), dict(new=0), dict(table=0), dict(lens=0), dict(slots=0), dict(B=0), dict(width=0), dict(most=-1), dict(nf=-1), dict(page=15), dict(page=24),
                dict(ctx=P + 2), dict(slots=P + 4), dict(info=P + 1), dict(lens=P), dict(lens=2 * P)):
        assert go(**bad) == snlp.ERR_ARG, bad
        assert "snlp_page_plan" in message()
    assert go(B=4097) == snlp.ERR_SHAPE
    assert go(most=(1 << 30) + 1) == snlp.ERR_SHAPE


def test_attention():
    n = C.c_size_t()

    def go(pl=None, out=P, ws=P, size=1 << 40, **kw):
        return lib.snlp_kv4_attention(C.byref(pl or pool()), C.byref(attn(**kw)), C.c_void_p(out), C.c_void_p(ws), C.c_size_t(size), None)
    for bad in (dict(q=None), dict(block_table=None), dict(lens=None), dict(out=0), dict(dtype=2), dict(B=0), dict(n_rows=-1), dict(n_head=3), dict(n_head=0),
                dict(n_rows=3), dict(max_pages=0), dict(max_len=-1), dict(q=P + 1), dict(out=P + 1), dict(lens=P + 2), dict(cu_q=P + 1), dict(q_token_stride=-1),
                dict(scale=float("nan")), dict(tile_rows=1), dict(tile_rows=-2), dict(tile_rows=32), dict(ws=P + 4), dict(dtype=0, q=P + 2)):
        assert go(**bad) == snlp.ERR_ARG, bad
        assert "snlp_kv4_attention" in message()
    assert go(B=4097, n_rows=4097) == snlp.ERR_SHAPE
    assert go(max_pages=1 << 28) == snlp.ERR_SHAPE
    assert go(n_rows=1 << 30, B=2, n_head=4) == snlp.ERR_SHAPE
    # a workspace that is missing or too small
    assert lib.snlp_kv4_attention_workspace(C.byref(pool(pages=None)), C.byref(attn(max_pages=100)), C.byref(n)) == 0 and n.value == 2 * 4 * 25 * 68 * 4
    assert go(max_pages=100, ws=0, size=0) == snlp.ERR_ARG and str(n.value) in message()
    assert go(max_pages=100, size=n.value - 1) == snlp.ERR_ARG
    assert lib.snlp_kv4_attention_workspace(C.byref(pool(pages=None)), C.byref(attn(max_pages=100, max_len=128)), C.byref(n)) == 0 and n.value == 0
    assert lib.snlp_kv4_attention_workspace(C.byref(pool()), C.byref(attn(n_head=3)), C.byref(n)) == snlp.ERR_ARG
    assert go(n_rows=0, q=None, out=0) == 0                  # no row: nothing to do


def test_plan_operands_that_overlap():
    """Blocks read the lengths, the free list and its head while others write the results: they may not share memory."""
    at = dict(ctx=P, new=P + 64, free=P + 128, head=P + 192, table=2 * P, slots=3 * P, pos=4 * P, cu=5 * P, lens=6 * P, info=7 * P)

    def go(B=4097, **kw):
        a = {k: C.c_void_p(v) for k, v in {**at, **kw}.items()}
        return lib.snlp_page_plan(a["ctx"], a["new"], B, 16, a["free"], 4, a["head"], a["table"], 4, 8, a["slots"], a["pos"], a["cu"], a["lens"], a["info"], None)
    for bad in (dict(lens=P - 4), dict(lens=P + 4), dict(lens=P + 60), dict(info=P + 192), dict(info=P + 188), dict(pos=P + 100), dict(slots=P + 8), dict(cu=P + 136),
                dict(free=2 * P + 28), dict(head=7 * P + 4), dict(table=P - 28), dict(ctx=4 * P + 28)):
        assert go(B=2, **bad) == snlp.ERR_ARG and "overlaps" in message(), bad


def test_read_into_rows_that_overlap():
    go = lambda st, v=2 * P, n=2, **kw: lib.snlp_kv4_read(C.byref(pool(**kw)), C.c_void_p(P), C.c_void_p(v), 1, (C.c_int64 * 4)(*st), C.c_void_p(P), n, None)  # noqa: E731
    for bad in ((0, 64, 128, 64), (128, 0, 128, 64), (128, 64, 63, 64), (128, 64, 128, 32)):
        assert go(bad) == snlp.ERR_ARG and "overlap" in message(), bad
    assert go((128, 64, 128, 64), v=P) == snlp.ERR_ARG and "overlap" in message()
    assert go((0, 63, 0, 64), n=1) == snlp.ERR_ARG                            # one token, two heads


@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan")])
def test_scale_has_to_be_finite(scale):
    assert lib.snlp_kv4_attention(C.byref(pool()), C.byref(attn(scale=scale)), C.c_void_p(P), C.c_void_p(P), C.c_size_t(1 << 40), None) == snlp.ERR_ARG
    assert "scale" in message()
