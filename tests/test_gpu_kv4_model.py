"""A model on a 4-bit key/value cache: prefill, decode steps, solver options and draft-and-verify against the oracle with a
cache that rounds what it stores, and against one another bit for bit."""
import numpy as np
import pytest
import torch

from oracle import snlp_oracle as O
from paper_2605_17842_b200 import synth
from tests import kv4_ref as R
from tests.gpu_util import TOL, dev, make_model, trace_err

pytestmark = pytest.mark.gpu


class Rounding:
    """An array of the oracle's cache that keeps what the 4-bit format keeps of the rows assigned to it."""

    def __init__(self, a):
        self.a = a

    def __setitem__(self, at, rows):
        self.a[at] = R.values(np.asarray(rows, np.float64))

    def __getitem__(self, at):
        return self.a[at]


def oracle_cache(cfg, B, ctx):
    kv = O.LayerKV(cfg.n_layer, B, ctx, cfg.n_head, cfg.head_dim)
    kv.k, kv.v = Rounding(kv.k), Rounding(kv.v)
    return kv


BF16 = synth.ModelConfig(3, 256, 2, 128, 512, 512, 1, "bf16")
FP32 = synth.ModelConfig(3, 128, 2, 64, 256, 256, 1, "fp32")
MHC = synth.ModelConfig(3, 256, 2, 128, 512, 512, 3, "bf16")
GENERIC = synth.ModelConfig(3, 192, 3, 64, 320, 384, 1, "bf16")     # bf16, but not for the tensor-core path

# Where library and oracle hold a key or value that differs by rounding noise, a code may fall on the other side of a border:
# the cached element then differs by a whole step (a fifteenth of its group's range) on one of the two sides.  fp32: a few
# elements of a cache at most, bf16: about 2 * 2^-9 * |x| / step = one in a hundred, i.e. 0.03 of the rows' own size, averaged
# over the visible keys.  Both stay inside the bf16 bound of the states.
TOL4 = TOL["bf16"]


def run_steps(cfg, B, T, Ks, generic=False, solver=None):
    W = synth.make_weights(cfg, seed=7, std=0.05, embed_std=1.0)
    m = make_model(cfg, W, max_rows=max(64, B), max_batch=B, max_ctx=T + 16)
    if generic:
        m.set_flag(1, 1)
    kv, kv_o = m.kv_cache(B, T + 16, bits=4), oracle_cache(cfg, B, T + 16)
    ids = synth.make_ids(cfg, B, T, seed=2)
    tok = m.prefill(kv, dev(ids))
    logits = O.prefill(cfg, W, ids, kv_o)
    assert len(kv) == T
    tok = tok.cpu().numpy().astype(np.int32)
    top = np.sort(logits, -1)
    for b in range(B):       # the prompt's token, unless two logits are closer than the states are known
        assert logits[b, tok[b]] >= top[b, -1] - 0.25 * (top[b, -1] - top[b, 0])
    for K in Ks:
        m.decode_step(kv, dev(tok), K)
        got = m.copy_trace(B).cpu().numpy()
        h0 = O.embed(cfg, W, tok.reshape(B, 1))
        want = (O.forward_sequential(cfg, W, h0, kv_o, kv_o.len) if K == 0
                else O.forward_snlp(cfg, W, h0, K, O.MODE_IDN, kv_o, kv_o.len)[0])[:, :, 0]
        kv_o.len += 1
        err = trace_err(got, want, TOL4)
        assert err <= TOL4, (K, err)
        tok = synth.make_ids(cfg, B, 1, seed=50 + K)[:, 0].astype(np.int32)
    return m, kv


@pytest.mark.parametrize("cfg,B,T", [(BF16, 1, 5), (BF16, 2, 40), (BF16, 3, 150), (FP32, 2, 30), (GENERIC, 2, 70)])
def test_decode_steps_match_the_oracle(cfg, B, T):
    run_steps(cfg, B, T, (0, 1, 2, 0))


def test_decode_steps_of_a_large_batch(cfg=BF16):
    run_steps(cfg, 20, 18, (0, 2))       # more rows than the decode regime takes


def test_decode_steps_on_the_generic_kernels():
    run_steps(BF16, 2, 33, (0, 2), generic=True)


def test_hcn_steps_match_the_oracle():
    W = synth.make_weights(MHC, seed=7, std=0.05, embed_std=1.0)
    m = make_model(MHC, W, max_rows=64, max_batch=2, max_ctx=64)
    kv, kv_o = m.kv_cache(2, 64, bits=4), oracle_cache(MHC, 2, 64)
    ids = synth.make_ids(MHC, 2, 30, seed=2)
    m.prefill(kv, dev(ids))
    O.prefill(MHC, W, ids, kv_o)
    from paper_2605_17842_b200 import snlp
    for K in (0, 2):
        tok = synth.make_ids(MHC, 2, 1, seed=9 + K)[:, 0].astype(np.int32)
        m.decode_step(kv, dev(tok), K, snlp.MODE_HCN)
        h0 = O.embed(MHC, W, tok.reshape(2, 1))
        want = O.forward_sequential(MHC, W, h0, kv_o, kv_o.len) if K == 0 else O.forward_snlp(MHC, W, h0, K, O.MODE_HCN, kv_o, kv_o.len)[0]
        kv_o.len += 1
        err = trace_err(m.copy_trace(2).cpu().numpy(), want[:, :, 0], TOL4)
        assert err <= TOL4, (K, err)


@pytest.mark.parametrize("cfg", [BF16, FP32, GENERIC])
@pytest.mark.parametrize("T", [20, 300])
def test_all_sweeps_equal_sequential_execution_bit_for_bit(cfg, T):
    W = synth.make_weights(cfg, seed=3, std=0.05, embed_std=1.0)
    m = make_model(cfg, W, max_rows=320, max_batch=2, max_ctx=T + 8)
    kv = m.kv_cache(2, T + 8, bits=4)
    m.prefill(kv, dev(synth.make_ids(cfg, 2, T, seed=4)))
    tok = dev(synth.make_ids(cfg, 2, 1, seed=5)[:, 0].astype(np.int32))
    a = m.decode_step(kv, tok, 0)
    seq = m.copy_trace(2)
    kv.truncate(T)
    b = m.decode_step(kv, tok, cfg.n_layer)
    assert torch.equal(m.copy_trace(2), seq) and torch.equal(a, b)


@pytest.mark.parametrize("cfg", [BF16, FP32])
@pytest.mark.parametrize("T,block,K", [(17, 4, 2), (250, 7, 1), (300, 14, 2)])
def test_draft_and_verify_emits_the_sequential_stream(cfg, T, block, K):
    W = synth.make_weights(cfg, seed=3, std=0.05, embed_std=1.0)
    n = 30
    m = make_model(cfg, W, max_rows=64, max_ctx=T + n + 2 * block + 4)
    ids = dev(synth.make_ids(cfg, 1, T, seed=4))

    def stream(run):
        kv = m.kv_cache(1, T + n + 2 * block + 4, bits=4)
        first = m.prefill(kv, ids)
        return run(kv, first)

    def sequential(kv, t):
        out = []
        for _ in range(n):
            t = m.decode_step(kv, t, 0)
            out.append(int(t))
        return out

    def spec(kv, t):
        out = []
        while len(out) < n:
            out += m.draft_and_verify(kv, t, block, K)[0]
            assert len(kv) == T + len(out)
        return out[:n]

    def spec_async(kv, t):
        out = []
        while len(out) < n:
            e, c = m.draft_and_verify_async(kv, t, block, K)
            out += e[:int(c[0])].tolist()
        assert len(kv) == T + len(out)
        return out[:n]

    def host(kv, t):
        t, out = t.cpu(), []
        for _ in range(n):
            t = m.decode_step_host(kv, t, 0)
            out.append(int(t))
        return out
    want = stream(sequential)
    assert len(set(want)) > 3
    assert stream(spec) == want
    assert stream(spec_async) == want
    assert stream(host) == want
    m.set_flag(0, 0)                       # without graphs
    assert stream(sequential) == want
    m.set_flag(0, 1)
    if cfg is BF16:
        m.set_flag(5, 0)                   # without the chained launch
        assert stream(sequential) == want


def test_solver_options_and_chunked_prefill():
    """Prefix, fwd initialisation and fused chunks run on the cache; a prompt in pieces leaves the states of one in a whole
    (up to the order of its attention's sums)."""
    from paper_2605_17842_b200 import snlp
    W = synth.make_weights(BF16, seed=3, std=0.05, embed_std=1.0)
    whole, parts = make_model(BF16, W, max_rows=128, max_ctx=128), make_model(BF16, W, max_rows=20, max_ctx=128)
    ids = dev(synth.make_ids(BF16, 1, 90, seed=4))
    tok = dev(np.array([17], np.int32))
    traces = []
    for m in (whole, parts):
        kv = m.kv_cache(1, 128, bits=4)
        m.prefill(kv, ids)
        m.decode_step(kv, tok, 0)
        traces.append(m.copy_trace(1).cpu().numpy())
    assert trace_err(traces[0], traces[1].astype(np.float64), TOL4) <= TOL4
    kv = whole.kv_cache(1, 128, bits=4)
    whole.prefill(kv, ids)
    for sol, equal in ((snlp.Solver(2, snlp.MODE_IDN, 1, snlp.INIT_H0, 1), True), (snlp.Solver(2, snlp.MODE_IDN, 0, snlp.INIT_FWD, 1), True),
                       (snlp.Solver(1, snlp.MODE_IDN, 0, snlp.INIT_H0, 3), False)):
        kv.truncate(90)
        whole.decode_step_solver(kv, tok, sol)
        tr = whole.copy_trace(1)
        assert torch.isfinite(tr[-1]).all()
        if equal:      # prefix 1 + two sweeps, or fwd + two sweeps, of three layers: exact
            assert torch.equal(tr.cpu(), torch.from_numpy(traces[0]))


def test_one_graph_serves_every_length():
    W = synth.make_weights(BF16, seed=3, std=0.05, embed_std=1.0)
    m = make_model(BF16, W, max_rows=64, max_ctx=700)
    kv = m.kv_cache(1, 700, bits=4)
    t = m.prefill(kv, dev(synth.make_ids(BF16, 1, 250, seed=4)))
    for _ in range(20):
        t = m.decode_step(kv, t, 2)
    assert m.graph_count() == 1 and len(kv) == 270
    kv.close()
    m.decode_step(m_kv := m.kv_cache(1, 64, bits=4), t, 2)
    assert m.graph_count() == 2 and len(m_kv) == 1


def test_refusals():
    from paper_2605_17842_b200 import snlp
    W = synth.make_weights(BF16, seed=3)
    m = make_model(BF16, W, max_rows=16, max_batch=2, max_ctx=32)
    for B, ctx, code in ((3, 32, snlp.ERR_SHAPE), (1, 33, snlp.ERR_SHAPE), (0, 8, snlp.ERR_ARG), (1, 0, snlp.ERR_ARG)):
        with pytest.raises(snlp.SnlpError) as e:
            m.kv_cache(B, ctx, bits=4)
        assert e.value.code == code
    with pytest.raises(snlp.SnlpError):
        m.kv_cache(1, 8, bits=8)
    tiny = make_model(synth.CONFIGS["tiny"], synth.make_weights(synth.CONFIGS["tiny"]), max_rows=8)
    with pytest.raises(snlp.SnlpError) as e:
        tiny.kv_cache(1, 8, bits=4)          # head_dim 32
    assert e.value.code == snlp.ERR_UNSUPPORTED
    kv = m.kv_cache(1, 32, bits=4)
    m.prefill(kv, dev(np.zeros((1, 32), np.int32)))
    with pytest.raises(snlp.SnlpError) as e:
        m.decode_step(kv, dev(np.zeros(1, np.int32)), 0)
    assert e.value.code == snlp.ERR_SHAPE
    m.close()
    with pytest.raises(snlp.SnlpError):
        kv.truncate(0)
    kv.close()


def test_a_new_cache_is_ready_for_any_stream():
    """A prompt on a stream that does not wait for the default one, right after a large cache was made: its pages and the
    unpacked rows have been cleared before, not while it runs."""
    W = synth.make_weights(BF16, seed=3, std=0.05, embed_std=1.0)
    m = make_model(BF16, W, max_rows=400, max_batch=8, max_ctx=1 << 18)
    ids = dev(synth.make_ids(BF16, 8, 50, seed=4))
    want = m.prefill(kv := m.kv_cache(8, 64, bits=4), ids).clone()
    trace = m.copy_trace(400).clone()
    kv.close()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        kv = m.kv_cache(8, 1 << 18, bits=4)
        with torch.cuda.stream(side):
            got = m.prefill(kv, ids)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(m.copy_trace(400), trace)
        kv.close()
