"""The 8-bit products' sums against float64, with bounds that one lost block or one lost bit would break (qsums)."""
import numpy as np
import pytest

import qref
import qsums
from sdcase import say

pytestmark = pytest.mark.gpu


def t(a, dtype=None):
    import torch
    x = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return x if dtype is None else x.to(dtype)


def dt(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def host(x):
    import torch
    if x.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu):
        return x.view(torch.uint8).cpu().numpy()
    return x.double().cpu().numpy()


def operands(M, N, K, spread=1.0):
    """Rows and a weight: their values, and what the calls take."""
    import torch
    from paper_2510_11331_amd import LinearQ
    r = np.random.default_rng([M, N, K])
    c, E = qref.quantise_rows(r.normal(size=(M, K)) * np.exp(spread * r.normal(size=(M, 1))))
    wc, wE = qref.quantise_weight(0.02 * r.normal(size=(N, K)) * np.exp(r.normal(size=(N, 1))))
    a, w = qref.row_values(c, E, K), qref.weight_values(wc, wE)
    return a, w, t(c).view(torch.float8_e4m3fn), t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu), LinearQ(t(qref.pack(wc, wE)), N, K)


def check_linear(M, N, K, dtype, fast=False):
    from paper_2510_11331_amd import linear_q
    a, w, q, e, wq = operands(M, N, K)
    want, s = qsums.terms(a, w)
    assert qsums.product_ok(host(linear_q(q, e, wq, dtype=dt(dtype), fast=fast)), want, qsums.sum_error(K, s), dtype)


def check_gate_up(M, F, K, fast=False):
    from paper_2510_11331_amd import gate_up_q
    a, w, q, e, wq = operands(M, 2 * F, K, 0.5)
    p, s = qsums.terms(a, w)
    h, err = qref.swiglu(p), qsums.swiglu_error(p, qsums.sum_error(K, s))
    got = [host(x) for x in gate_up_q(q, e, wq, fast=fast)]
    blocks = -(-F // 128)
    E = got[1][:, :blocks].astype(np.int64)
    assert not got[0][:, F:].any() and not got[1][:, blocks:].any()
    hc, hE = qref.quantise_rows(h)
    scale = np.repeat(2.0 ** (np.maximum(E, hE) - 127.0), 128, 1)[:, :F]
    assert qsums.codes_ok(qref.row_values(got[0], E, F), h, err, qref.row_values(hc, hE, F), scale)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(64, 300, 2000), (65, 300, 2000), (200, 520, 1100), (300, 1000, 4200), (1100, 1040, 600)])
def test_sums_of_any_rows(M, N, K, dtype):
    """Sums are as exact above 64 rows as below, for both types."""
    say("linear sums", M, N, K, dtype)
    check_linear(M, N, K, dtype)


@pytest.mark.parametrize("M,F,K", [(64, 272, 2000), (65, 272, 2000), (200, 1040, 1100), (320, 528, 4200), (1100, 528, 600)])
def test_gate_up_sums_of_any_rows(M, F, K):
    say("gate_up sums", M, F, K)
    check_gate_up(M, F, K)


@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("M,K", [(1, 16384), (1, 16512), (3, 28672), (64, 16500), (64, 40000)])
def test_sums_of_few_rows_long_k(M, K, fast):
    """Up to 64 rows every sum is exact, also where K is past what the streaming kernel holds scales of."""
    say("few rows, long K", M, K, fast)
    for dtype in ("fp32", "bf16"):
        check_linear(M, 200, K, dtype, fast)
    check_gate_up(M, 144, K, fast)
