"""The 8-bit feed-forward operators without a GPU: the format's reference, and what the calls refuse before they enqueue
anything."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import qref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2510_11331_amd", "libsd.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libsd.so not built (run __graft_entry__.build())")


def test_reference_codes_are_torchs():
    v = np.concatenate([np.random.default_rng(1).normal(0, s, 4000) for s in (1e-3, 0.1, 30.0, 140.0)])
    v = np.concatenate([v, qref.POS, (qref.POS[1:] + qref.POS[:-1]) / 2, [0.0, -0.0]]).astype(np.float32)
    v = v[np.abs(v) <= 448]
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(qref.code(v), want)
    assert np.array_equal(qref.value(want), torch.from_numpy(want).view(torch.float8_e4m3fn).double().numpy())


def test_reference_exponents():
    for a, E in ((0.0, 1), (1e-45, 1), (448.0, 127), (np.nextafter(448.0, 449.0), 128), (224.0, 126), (1.75, 119), (1.7500001, 120),
                 (3.4e38, 247), (448 * 2.0 ** -126, 1), (449 * 2.0 ** -126, 2)):
        assert qref.exponent(np.array(a)) == E, a


def test_reference_round_trip():
    r = np.random.default_rng(2)
    y = r.normal(size=(5, 300)) * np.exp(r.normal(size=(5, 1)))
    c, E = qref.quantise_rows(y)
    v = qref.row_values(c, E, 300)
    scale = np.repeat(2.0 ** (E - 127.0), 128, 1)[:, :300]
    # half a step: 2^-4 of a normal code, 2^-10 scales of a subnormal one
    assert (np.abs(v - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * scale)).all()
    assert c.shape == (5, 384) and not c[:, 300:].any()


@needs_lib
def test_sizes():
    from paper_2510_11331_amd._lib import lib
    L = lib()
    for N, K in ((1, 1), (16, 128), (17, 129), (22016, 4096), (1000, 1000), (1 << 22, 1 << 18)):
        assert L.sd_linear_q_bytes(N, K) == qref.up(N, 16) * qref.up(K, 128) + -(-N // 128) * qref.up(-(-K // 128), 4)
    for N, K in ((0, 1), (1, 0), (-1, 5), (1, (1 << 18) + 1), ((1 << 22) + 1, 1)):
        assert L.sd_linear_q_bytes(N, K) == 0
    assert L.sd_gate_up_q_workspace_bytes(40, 11008, 4096) == 40 * 11008 * 4 and L.sd_gate_up_q_workspace_bytes(0, 16, 1) == 0
    for M, F, K in ((-1, 16, 1), (1, 0, 1), (1, 8, 1), (1, 24, 1), (1 << 23, 16, 1), (1, 16, 0), (1, (1 << 18) + 16, 1)):
        assert L.sd_gate_up_q_workspace_bytes(M, F, K) == 0
    # K ranges: whole sums [ranges, M, N rounded up to 4]
    assert L.sd_linear_q_workspace_bytes(100, 1023, 11008) in (2 * 100 * 1024 * 4, 4 * 100 * 1024 * 4)
    assert L.sd_linear_q_workspace_bytes(-1, 1, 1) == L.sd_linear_q_workspace_bytes(1, 0, 1) == L.sd_linear_q_workspace_bytes(0, 1, 1) == 0


@needs_lib
def test_calls_refuse():
    """The pointers are never dereferenced."""
    from paper_2510_11331_amd import _lib
    L, E, A = _lib.lib(), _lib.SD_EINVAL, 1 << 20
    BF, F32 = _lib.SD_DTYPE_BF16, _lib.SD_DTYPE_F32

    pk = dict(src=A, dst=A, N=64, K=64, dtype=BF)
    for bad in (dict(src=None), dict(dst=None), dict(N=0), dict(K=0), dict(K=(1 << 18) + 1), dict(dtype=2), dict(dtype=-1), dict(src=A + 1),
                dict(dst=A + 8), dict(src=A + 2, dtype=F32)):
        assert L.sd_pack_linear_q(*{**pk, **bad}.values(), None) == E, bad

    nm = dict(M=2, d=64, dtype=F32, x=A, n_add=1, add=A, x_out=A, gain=A, gain_dtype=BF, eps=1e-5, q=A, exps=A)
    for bad in (dict(M=-1), dict(d=0), dict(d=16385), dict(dtype=2), dict(gain_dtype=2), dict(n_add=-1), dict(n_add=7), dict(eps=0.0),
                dict(eps=float("nan")), dict(x=None), dict(add=None), dict(x_out=None), dict(gain=None), dict(q=None), dict(exps=None),
                dict(x=A + 2), dict(add=A + 2), dict(x_out=A + 1), dict(gain=A + 1), dict(q=A + 8)):
        assert L.sd_add_rmsnorm_q(*{**nm, **bad}.values(), None) == E, bad
    assert L.sd_add_rmsnorm_q(*{**nm, "M": 0, "x": None, "q": None}.values(), None) == _lib.SD_OK

    n = L.sd_linear_q_workspace_bytes(100, 64, 11008)
    assert n >= 2 * 100 * 64 * 4
    ln = dict(M=100, N=64, K=11008, q=A, exps=A, w=A, add=A, out=A, ldo=64, dtype=F32, ws=A, n=n)
    for bad in (dict(M=-1), dict(N=0), dict(K=0), dict(K=(1 << 18) + 1), dict(q=None), dict(exps=None), dict(w=None), dict(out=None), dict(ldo=63),
                dict(dtype=2), dict(q=A + 8), dict(w=A + 8), dict(add=A + 2), dict(out=A + 2), dict(M=(1 << 22) + 1), dict(ws=None), dict(n=n - 1),
                dict(ws=A + 8), dict(exps=A + 2)):
        assert L.sd_linear_q(*{**ln, **bad}.values(), None) == E, bad
    assert L.sd_linear_q(*{**ln, "M": 0, "out": None}.values(), None) == _lib.SD_OK

    n = L.sd_gate_up_q_workspace_bytes(2, 64, 64)
    gu = dict(M=2, F=64, K=64, q=A, exps=A, w=A, q_out=A, exps_out=A, ws=A, n=n)
    for bad in (dict(M=-1), dict(F=0), dict(F=65), dict(F=72), dict(K=0), dict(q=None), dict(exps=None), dict(w=None), dict(q_out=None),
                dict(exps_out=None), dict(ws=None), dict(n=n - 1), dict(q=A + 8), dict(w=A + 8), dict(q_out=A + 8), dict(ws=A + 8), dict(exps=A + 2)):
        assert L.sd_gate_up_q(*{**gu, **bad}.values(), None) == E, bad
    assert L.sd_gate_up_q(*{**gu, "M": 0, "q": None}.values(), None) == _lib.SD_OK


@needs_lib
def test_python_refuses():
    """Shapes, types and layouts (host tensors: none of these calls gets as far as needing a GPU)."""
    from paper_2510_11331_amd import LinearQ, add_rmsnorm_q, gate_up_q, linear_q, pack_linear_q
    x, g = torch.zeros(3, 64), torch.ones(64)

    def refused(f, *a, **k):
        with pytest.raises(ValueError):
            f(*a, **k)

    refused(pack_linear_q, torch.zeros(4, 4))                                 # a host tensor
    refused(pack_linear_q, torch.zeros(4, 4, dtype=torch.float16))
    refused(pack_linear_q, torch.zeros(4, 8)[:, ::2])
    refused(pack_linear_q, torch.zeros(4))
    refused(pack_linear_q, torch.zeros(0, 4))
    refused(add_rmsnorm_q, x, g, 1e-5)                                        # a host tensor
    for kw in (dict(add=torch.zeros(3, 63)), dict(add=torch.zeros(7, 3, 64)), dict(add=torch.zeros(3, 64).bfloat16()),
               dict(add=torch.zeros(64, 3).t()), dict(add=x, x_out=torch.zeros(3, 65)), dict(x_out=torch.zeros(3, 64))):
        refused(add_rmsnorm_q, x, g, 1e-5, **kw)
    refused(add_rmsnorm_q, x, g[:63], 1e-5)
    refused(add_rmsnorm_q, x.half(), g, 1e-5)
    refused(add_rmsnorm_q, torch.zeros(1, 16385), torch.zeros(16385), 1e-5)
    with pytest.raises(ValueError):
        LinearQ(torch.zeros(17, dtype=torch.uint8), 4, 4)
    w = LinearQ(torch.zeros(16 * 128 + 4, dtype=torch.uint8), 16, 64)
    q, e = torch.zeros(3, 128).to(torch.float8_e4m3fn), torch.zeros(3, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    assert w.codes.shape == (2048,) and w.exps.shape == (1, 4)
    refused(linear_q, q, e, w)                                                # host tensors
    refused(linear_q, q[:, :64], e, w)
    refused(linear_q, q, e[:2], w)
    refused(linear_q, q.float(), e, w)
    refused(linear_q, q, e, w, dtype=torch.float16)
    refused(linear_q, q, e, w, out=torch.zeros(3, 15))
    refused(linear_q, q, e, w, out=torch.zeros(16, 3).t())
    refused(linear_q, q, e, w, out=torch.zeros(1, 16).expand(3, 16))
    refused(linear_q, q, e, w, add=torch.zeros(3, 16).bfloat16())
    refused(linear_q, q, e, w, add=torch.zeros(3, 32)[:, :16])
    refused(gate_up_q, q, e, w)                                               # 16 rows are no gate and up block


@needs_lib
def test_model_dtype():
    """SD_DTYPE_BF16_FFN_Q: sizes of a configuration, its plan queries, and the binding's refusal of fp32 models."""
    import synth
    from paper_2510_11331_amd import _lib
    from paper_2510_11331_amd.engine import model_cfg
    L = _lib.lib()
    c = _lib.Config()
    t, d = synth.MODELS["small_target"], synth.MODELS["small_draft"]
    c.target, c.draft = model_cfg(t), model_cfg(d)
    c.max_slots, c.max_batch, c.gamma_max, c.max_ctx = 4, 2, 4, 128
    c.kv_block, c.kv_blocks_target, c.kv_blocks_draft, c.prefill_rows, c.temperature = 16, 32, 32, 128, 1.0
    plain, pool = L.sd_workspace_bytes(C.byref(c)), L.sd_kv_pool_bytes(C.byref(c), 0)
    c.target = model_cfg(t, ffn_q=True)
    assert c.target.dtype == _lib.SD_DTYPE_BF16_FFN_Q
    assert L.sd_workspace_bytes(C.byref(c)) > plain and L.sd_kv_pool_bytes(C.byref(c), 0) == pool
    p = _lib.ProjPlan()
    plan = lambda proj: L.sd_plan_projection(C.byref(c), _lib.SD_PASS_VERIFY, proj, 10, C.byref(p))
    assert plan(_lib.SD_PROJ_QKV) == plan(_lib.SD_PROJ_O) == plan(_lib.SD_PROJ_LM_HEAD) == _lib.SD_OK
    assert plan(_lib.SD_PROJ_GATEUP) == plan(_lib.SD_PROJ_DOWN) == _lib.SD_EINVAL
    c.target.dtype = 3
    assert L.sd_workspace_bytes(C.byref(c)) == 0
    c.target = model_cfg(synth.ModelShape(1, 16384, 128, 128, 16384, t.vocab, "bf16"), ffn_q=True)
    assert L.sd_workspace_bytes(C.byref(c)) > 0
    c.target = model_cfg(synth.ModelShape(1, 16512, 129, 129, 16384, t.vocab, "bf16"), ffn_q=True)    # rows past what the norm holds
    assert L.sd_workspace_bytes(C.byref(c)) == 0
    with pytest.raises(ValueError):
        model_cfg(synth.MODELS["tiny_target"], ffn_q=True)
