"""That the checks of the 8-bit products' GPU tests see what they are for: mistakes planted in the operands, on the CPU."""
import numpy as np
import pytest

import qplans
import qref
import qsums


def example(K, M=20, N=64):
    r = np.random.default_rng(K)
    c, E = qref.quantise_rows(r.normal(size=(M, K)) * np.exp(0.5 * r.normal(size=(M, 1))))
    wc, wE = qref.quantise_weight(r.normal(size=(N, K)) / np.sqrt(K))
    return qref.row_values(c, E, K), qref.weight_values(wc, wE)


def mistakes(a, w):
    """Operands as a wrong kernel would have read them, in one tile of 16 rows or for all."""
    K = a.shape[1]
    last, mid = (K - 1) // 128 * 128, (K // 2) // 128 * 128

    def change(name, x, k, f, rows=slice(None)):
        y = x.copy()
        y[rows, k] = f(y[rows, k])
        return name, y

    yield change("a block of 16 rows is lost", a, slice(mid, mid + 128), lambda v: 0 * v, slice(0, 16))
    yield change("the last block is lost", a, slice(last, K), lambda v: 0 * v)
    yield change("the last entry is lost", a, slice(K - 1, K), lambda v: 0 * v)
    yield change("a block has twice its scale", a, slice(mid, mid + 128), lambda v: 2 * v, slice(0, 16))
    if K >= 256:
        yield change("a block is read twice", a, slice(128, 256), lambda v: a[:16, :128], slice(0, 16))


@pytest.mark.parametrize("K", sorted({c[6] for c in qplans.LINEAR + qplans.GATE_UP} | {128, 16500, 40000}))
def test_checks_see_mistakes(K):
    """At every K of the GPU cases: sums in float32 pass, those of wrong operands do not."""
    a, w = example(K)
    want, s = qsums.terms(a, w)
    for err, sloppy in ((qsums.sum_error(K, s), 0.0), (qsums.cut_error(s), 2e-5)):
        noise = sloppy * s * np.random.default_rng(1).normal(size=s.shape)
        plain = (a.astype(np.float32) @ w.T.astype(np.float32)).astype(np.float64) + noise
        assert qsums.product_ok(plain.astype(np.float32).astype(np.float64), want, err, "fp32")
        assert qsums.product_ok(qsums.to_bf16(plain), want, err, "bf16")
        assert codes_ok(plain, want, err)
        for name, b in mistakes(a, w):
            wrong = b @ w.T
            assert not qsums.product_ok(wrong.astype(np.float32).astype(np.float64), want, err, "fp32"), name
            assert not qsums.product_ok(qsums.to_bf16(wrong), want, err, "bf16"), name
            assert not codes_ok(wrong, want, err), name
    # exact sums: the 8-bit instruction's cut is seen too
    cut = want + 2e-5 * s * np.random.default_rng(2).normal(size=s.shape)
    assert not qsums.product_ok(cut, want, qsums.sum_error(K, s), "fp32")


def codes_ok(product, want, err):
    h, F = qref.swiglu(want), want.shape[1] // 2
    (c, E), (hc, hE) = qref.quantise_rows(qref.swiglu(product)), qref.quantise_rows(h)
    scale = np.repeat(2.0 ** (np.maximum(E, hE) - 127.0), 128, 1)[:, :F]
    return qsums.codes_ok(qref.row_values(c, E, F), h, qsums.swiglu_error(want, err), qref.row_values(hc, hE, F), scale)


def test_rounding_to_bf16():
    import torch
    v = np.random.default_rng(3).normal(size=4000) * 2.0 ** np.random.default_rng(4).integers(-60, 60, size=4000)
    v = np.concatenate([v, [0.0, 1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -1 - 2.0 ** -8]])
    v = v.astype(np.float32).astype(np.float64)
    assert np.array_equal(qsums.to_bf16(v), torch.from_numpy(v).to(torch.bfloat16).double().numpy())
