"""The 8-bit feed-forward operators against their definitions in float64 (qref)."""
import math

import numpy as np
import pytest

import qref
from sdcase import say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24       # half a step of fp32, of bf16 2^-8, relative


def t(a, dtype=None):
    import torch
    x = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return x if dtype is None else x.to(dtype)


def host(x):
    import torch
    if x.dtype in (torch.float8_e4m3fn, torch.float8_e8m0fnu):
        return x.view(torch.uint8).cpu().numpy()
    return x.double().cpu().numpy()


def dt(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def same_codes(a, b):
    """Equal bytes, or both NaN."""
    return ((a == b) | ((a & 127 == 127) & (b & 127 == 127))).all()


def rows8(r, M, K, spread=1.0):
    """Codes and exponents of random rows, and their tensors."""
    import torch
    y = r.normal(size=(M, K)) * np.exp(spread * r.normal(size=(M, 1)))
    c, E = qref.quantise_rows(y)
    return c, E, t(c).view(torch.float8_e4m3fn), t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu)


def weight8(r, N, K):
    import torch
    from paper_2510_11331_amd import LinearQ
    w = 0.02 * r.normal(size=(N, K)) * np.exp(r.normal(size=(N, 1)))
    c, E = qref.quantise_weight(w)
    return c, E, LinearQ(t(qref.pack(c, E)), N, K)


def product64(c, E, wc, wE):
    """The product and the sum of its terms' magnitudes."""
    a, w = qref.row_values(c, E, wc.shape[1]), qref.weight_values(wc, wE)
    return a @ w.T, np.abs(a) @ np.abs(w).T


def sum_error(K, mag):
    """What fp32 sums of K exact terms may be off by: at most K + K / 128 + 16 additions (the terms, the blocks, the waves),
    each off by at most a step (2 U32: the matrix unit may cut instead of rounding) of a partial sum that `mag` bounds."""
    return (K + K / 128 + 16) * 2 * U32 * mag


# ------------------------------------------------------------------ packing


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (130, 257), (33, 4), (300, 1000), (1000, 384), (2, 6), (144, 514)])
def test_pack(N, K, dtype):
    from paper_2510_11331_amd import pack_linear_q
    say("pack", N, K, dtype)
    r = np.random.default_rng([N, K])
    w = t((0.02 * r.normal(size=(N, K)) * np.exp(2 * r.normal(size=(N, 1)))).astype(np.float32), dt(dtype))
    got = pack_linear_q(w)
    assert np.array_equal(got.data.cpu().numpy(), qref.pack(*qref.quantise_weight(host(w))))
    assert got.codes.numel() + got.exps.numel() == got.data.numel()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pack_special_values(dtype):
    """Blocks of zeros, of the type's smallest and largest numbers, at the scale's border, with NaN and infinities, with
    ties; an unaligned source."""
    import torch
    from paper_2510_11331_amd import pack_linear_q
    say("pack special", dtype)
    r = np.random.default_rng(5)
    w = r.normal(size=(128, 128 * 9)).astype(np.float32)
    big = 3.38e38
    w[:, :128] = 0
    w[:, 128:256] *= 1e-38                                  # smaller than the smallest scale reaches
    w[:, 256:384] *= big / 8
    w[3, 256] = big
    w[:, 384:512] = np.clip(w[:, 384:512], -1, 1) * 440
    w[0, 384] = 448.0                                       # border: stays in the smaller scale
    w[:, 512:640] = np.clip(w[:, 512:640], -1, 1) * 440
    w[0, 512] = 450.0                                       # representable in bf16, past the border
    w[5, 640], w[6, 641], w[7, 642] = np.nan, np.inf, -np.inf
    w[:, 768:896] = np.nan
    w[:, 896:1024] = r.integers(-511, 512, size=(128, 128))     # ties
    src = t(w, dt(dtype))
    want = qref.pack(*qref.quantise_weight(host(src)))
    got = pack_linear_q(src).data.cpu().numpy()
    n = 128 * 128 * 9
    assert same_codes(got[:n], want[:n]) and np.array_equal(got[n:], want[n:])
    flat = torch.empty(src.numel() + 1, dtype=src.dtype, device="cuda")
    flat[1:] = src.view(-1)
    got = pack_linear_q(flat[1:].view(src.shape)).data.cpu().numpy()
    assert same_codes(got[:n], want[:n]) and np.array_equal(got[n:], want[n:])


# ------------------------------------------------------------------ norm


def check_norm(x, add, gain, eps, xo, q, exps):
    """x_out is the sum rounded once (and for bf16 through fp32); the codes are those of the normed row in fp32.  The
    reference's y and the kernel's, both in 64 bits, are a few 2^-53 apart; where y lies that near (2^-48) to where its
    code or its block's exponent changes, either is right."""
    import torch
    x64 = host(x)
    if add is not None:
        s = x64 + host(add).reshape(-1, *x64.shape).sum(0)
        want = torch.from_numpy(s).to(x.dtype).double().numpy()
        assert np.array_equal(host(xo), want, equal_nan=True)
        x64 = want
    with np.errstate(all="ignore"):
        y = qref.norm(x64, host(gain)[None], float(np.float32(eps)))
        ways = [qref.quantise_rows((y * f).astype(np.float32).astype(np.float64)) for f in (1.0, 1 - 2.0 ** -48, 1 + 2.0 ** -48)]
    gc, ge = host(q), host(exps)
    blocks = ways[0][1].shape[1]
    assert not ge[:, blocks:].any() and gc.shape[1] == 128 * blocks
    ok = np.zeros(ge[:, :blocks].shape, dtype=bool)
    for c, E in ways:
        same = ((gc == c) | ((gc & 127 == 127) & (c & 127 == 127))).reshape(*E.shape, 128)
        near = [((gc == c2) | ((gc & 127 == 127) & (c2 & 127 == 127))).reshape(*E.shape, 128) & (E2 == E)[..., None] for c2, E2 in ways]
        ok |= (ge[:, :blocks] == E) & (same | near[0] | near[1] | near[2]).all(-1)
    assert ok.all(), np.argwhere(~ok)[:5]


@pytest.mark.parametrize("dtype,gain_dtype", [("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("M,d,n_add", [(1, 1, 0), (3, 64, 1), (5, 129, 2), (2, 1000, 6), (7, 1024, 3), (4, 2816, 1), (40, 4096, 4),
                                       (3, 5120, 6), (2, 8190, 5), (2, 8192, 2), (2, 8196, 2), (3, 16384, 6), (1, 16383, 1), (2, 2049, 0)])
def test_norm(M, d, n_add, dtype, gain_dtype):
    from paper_2510_11331_amd import add_rmsnorm_q
    say("norm", M, d, n_add, dtype, gain_dtype)
    r = np.random.default_rng([M, d, n_add])
    x = t((r.normal(size=(M, d)) * np.exp(2 * r.normal(size=(M, 1)))).astype(np.float32), dt(dtype))
    add = t(r.normal(size=(n_add, M, d)).astype(np.float32), dt(dtype)) if n_add else None
    if n_add == 1:
        add = add[0]
    gain = t((1 + 0.1 * r.normal(size=d)).astype(np.float32), dt(gain_dtype))
    keep = x.clone()
    xo, q, e = add_rmsnorm_q(x, gain, 1e-5, add=add)
    assert bool((x == keep).all()) and (xo is x) == (n_add == 0)
    check_norm(x, add, gain, 1e-5, xo, q, e)


def test_norm_special_rows():
    """Zero rows, rows of tiny and huge numbers, a NaN and an infinity (each row alone is affected), in place, and a row
    length that makes the last block partial."""
    import torch
    from paper_2510_11331_amd import add_rmsnorm_q
    say("norm special rows")
    r = np.random.default_rng(8)
    x = r.normal(size=(8, 300)).astype(np.float32)
    x[0] = 0
    x[1] *= 1e-30
    x[2] *= 1e18
    x[3, 299] = np.nan
    x[4, 7] = np.inf
    x[5] *= 1e30
    for name in ("fp32", "bf16"):
        xs = t(x, dt(name))
        gain = t((1 + 0.1 * r.normal(size=300)).astype(np.float32))
        add = torch.zeros_like(xs)
        add[7] = 1.0
        before = xs.clone()
        xo, q, e = add_rmsnorm_q(xs, gain, 1e-6, add=add, x_out=xs)
        assert xo is xs
        check_norm(before, add, gain, 1e-6, xo, q, e)
        nan = (host(q) & 127) == 127
        assert nan[3, :300].all() and nan[4, 7] and nan[4].sum() == 1 and not nan[[0, 1, 2, 5, 6, 7]].any() and not nan[:, 300:].any()


def test_norm_unaligned():
    """Rows that start on the type's own alignment only."""
    import torch
    from paper_2510_11331_amd import add_rmsnorm_q
    say("norm unaligned")
    r = np.random.default_rng(9)
    for name in ("fp32", "bf16"):
        flat = t(r.normal(size=5 * 256 + 1).astype(np.float32), dt(name))
        x = flat[1:].view(5, 256)
        gain = t(r.normal(size=257).astype(np.float32), torch.bfloat16)[1:]
        add = t(r.normal(size=(2, 5, 256)).astype(np.float32), dt(name))
        check_norm(x, add, gain, 1e-5, *add_rmsnorm_q(x, gain, 1e-5, add=add))


# ------------------------------------------------------------------ product

SHAPES = [(1, 1, 1), (1, 1000, 1000), (2, 16, 128), (5, 130, 129), (15, 64, 513), (16, 100, 640), (17, 48, 100), (33, 257, 700), (40, 512, 1024),
          (48, 96, 2816), (49, 33, 300), (64, 160, 256), (65, 144, 384), (130, 300, 520), (257, 129, 1100), (320, 640, 256)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(M, N, K, dtype):
    from paper_2510_11331_amd import linear_q
    say("linear", M, N, K, dtype)
    r = np.random.default_rng([M, N, K])
    c, E, q, e = rows8(r, M, K)
    wc, wE, w = weight8(r, N, K)
    want, mag = product64(c, E, wc, wE)
    got = host(linear_q(q, e, w, dtype=dt(dtype)))
    assert got.shape == want.shape
    check_product(got, want, mag, K, dtype)


# The 8-bit matrix instruction, which products of many rows run on where the caller chose it, drops low bits of the products it adds: probed
# at 2^-14 to 2^-16 of a sum's root mean square for any K; as a bound, 2^-12 of the terms' magnitudes
CUT8 = 2.0 ** -12


def check_product(got, want, mag, K, dtype):
    tol = sum_error(K, mag)
    if dtype == "bf16":
        tol = 2.0 ** -8 * np.abs(want) + (tol + CUT8 * mag) * (1 + 2.0 ** -8)
    assert (np.abs(got - want) <= tol).all(), np.abs((got - want) / np.maximum(tol, 1e-300)).max()


def test_linear_fp32_is_as_exact_as_fp32():
    """In the 2-norm, fp32 outputs are within 2^-20 of the product (the sums' own error, 2^-22 at these K)."""
    from paper_2510_11331_amd import linear_q
    say("linear accuracy")
    for M, N, K in ((8, 128, 4096), (100, 128, 4096), (300, 256, 2048)):
        r = np.random.default_rng(M)
        c, E, q, e = rows8(r, M, K)
        wc, wE, w = weight8(r, N, K)
        want, _ = product64(c, E, wc, wE)
        assert np.linalg.norm(host(linear_q(q, e, w)) - want) <= 2.0 ** -20 * np.linalg.norm(want)


@pytest.mark.parametrize("M", [1, 40, 200])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_linear_add_and_strides(M, dtype):
    """out and add as column ranges of wider buffers, at every alignment of the first column; what lies beside them stays."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("linear add", M, dtype)
    N, K = 77, 300
    r = np.random.default_rng(M)
    c, E, q, e = rows8(r, M, K)
    wc, wE, w = weight8(r, N, K)
    want, mag = product64(c, E, wc, wE)
    for off in (0, 1, 3, 4):
        wide = torch.full((M + 2, 96), 7.0, dtype=dt(dtype), device="cuda")
        addw = t(r.normal(size=(M + 2, 96)).astype(np.float32))
        out, add = wide[1:M + 1, off:off + N], addw[1:M + 1, off:off + N]
        got = linear_q(q, e, w, add=add, out=out)
        assert got is out
        a = host(add)
        check_product(host(got), want + a, mag + np.abs(a), K, dtype)
        wide[1:M + 1, off:off + N] = 7.0
        assert bool((wide == 7.0).all())
        if dtype == "fp32":                                   # in place
            x = addw.clone()
            linear_q(q, e, w, add=x[1:M + 1, off:off + N], out=x[1:M + 1, off:off + N])
            check_product(host(x[1:M + 1, off:off + N]), want + a, mag + np.abs(a), K, dtype)
            x[1:M + 1, off:off + N] = addw[1:M + 1, off:off + N]
            assert bool((x == addw).all())


@pytest.mark.parametrize("M", [3, 100])
def test_linear_special(M):
    """A NaN code makes NaN of its row's outputs and no others; far apart scales; a zero row; no rows."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("linear special", M)
    N, K = 40, 700
    r = np.random.default_rng(11)
    c, E, _, _ = rows8(r, M, K)
    wc, wE, w = weight8(r, N, K)
    c, E = c.copy(), E.copy()
    c[0] = 0
    E[0] = 1
    E[1] = [1, 254, 1, 100, 1, 200][:E.shape[1]]              # 2^-126 to 2^127
    c[1, :128] = c[1, 256:384] = 0
    c[1, 128:256] = 0
    c[2, 650] = 0x7f
    q = t(c).view(torch.float8_e4m3fn)
    for dtype in ("fp32", "bf16"):
        got = host(linear_q(q, t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu), w, dtype=dt(dtype)))
        assert np.isnan(got[2]).all() and not np.isnan(got[[0, 1, *range(3, M)]]).any() and not got[0].any()
        rows = [0, 1, *range(3, M)]
        want, mag = product64(c[rows], E[rows], wc, wE)
        with np.errstate(over="ignore"):
            assert np.isfinite(got[rows]).all()
        check_product(got[rows], want, mag, K, dtype)
    assert linear_q(q[:0], t(qref.exps_bytes(E[:0])).view(torch.float8_e8m0fnu), w).shape == (0, N)


def test_linear_offsets_past_32_bits():
    """An output of more than 2^32 entries: its first and last rows and columns."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("linear large")
    M, N, K = 65600, 65552, 64
    r = np.random.default_rng(12)
    c, E, q1, e1 = rows8(r, 64, K)
    wc, wE, w1 = weight8(r, 128, K)
    q, e = q1.view(torch.uint8).repeat(1025, 1).view(torch.float8_e4m3fn), e1.view(torch.uint8).repeat(1025, 1).view(torch.float8_e8m0fnu)
    from paper_2510_11331_amd import LinearQ
    wc2, wE2 = np.tile(wc, (513, 1))[:N], np.tile(wE, (513, 1))[:-(-N // 128)]
    w = LinearQ(t(qref.pack(wc2, wE2)), N, K)
    out = linear_q(q, e, w, dtype=torch.bfloat16)
    want, mag = product64(c, E, wc, wE)
    for i in (0, 32768, 65536):
        for j in (0, 32768, 65408):
            got = host(out[i:i + 64, j:j + 128])
            check_product(got, want, mag, K, "bf16")
    check_product(host(out[:64, N - 16:]), want[:, :16], mag[:, :16], K, "bf16")


# ------------------------------------------------------------------ gate/up


def check_codes_of(q, e, h, err):
    """(q, e) are codes of h known to +- err: the exponent is that of a maximum in the range, a value is within half a step
    (2^-4 of it, or 2^-10 scales below the smallest normal code) of a number in its range."""
    M, F = h.shape
    gc, ge = host(q), host(e).astype(np.int64)
    blocks = -(-F // 128)
    assert not ge[:, blocks:].any() and not gc[:, F:].any()
    pad = lambda a: np.pad(a, ((0, 0), (0, 128 * blocks - F))).reshape(M, blocks, 128)
    lo, hi = qref.exponent(pad(np.maximum(np.abs(h) - err, 0)).max(-1)), qref.exponent(pad(np.abs(h) + err).max(-1))
    assert ((lo <= ge[:, :blocks]) & (ge[:, :blocks] <= hi)).all()
    v = qref.row_values(gc, ge[:, :blocks], F)
    scale = np.repeat(2.0 ** (ge[:, :blocks] - 127.0), 128, 1)[:, :F]
    assert (np.abs(v - h) <= err + np.maximum(2.0 ** -4 * (np.abs(h) + err), 2.0 ** -10 * scale)).all()


def swiglu_error(p, tol):
    """What silu(g) u may be off by when g and u are off by tol, and by four fp32 roundings and an exponential good to 4 of
    them besides: |silu'| <= 1.1."""
    s = p.reshape(p.shape[0], -1, 2, 16)
    e = tol.reshape(p.shape[0], -1, 2, 16)
    g, u, dg, du = (a.reshape(p.shape[0], -1) for a in (s[:, :, 0], s[:, :, 1], e[:, :, 0], e[:, :, 1]))
    silu = np.abs(g / (1 + np.exp(-g)))
    return 1.1 * dg * (np.abs(u) + du) + silu * du + 8 * 2 * U32 * silu * np.abs(u)


@pytest.mark.parametrize("M,F,K", [(1, 16, 1), (1, 688, 256), (2, 128, 128), (5, 144, 300), (16, 256, 640), (40, 1024, 513), (48, 272, 128), (64, 400, 200),
                                   (65, 384, 300), (130, 272, 700), (300, 1040, 260)])
def test_gate_up(M, F, K):
    from paper_2510_11331_amd import gate_up_q
    say("gate_up", M, F, K)
    r = np.random.default_rng([M, F, K])
    c, E, q, e = rows8(r, M, K, 0.5)
    wc, wE, w = weight8(r, 2 * F, K)
    p, mag = product64(c, E, wc, wE)
    tol = sum_error(K, mag) + (CUT8 * mag if M > 64 else 0)
    check_codes_of(*gate_up_q(q, e, w), qref.swiglu(p), swiglu_error(p, tol))


# ------------------------------------------------------------------ together


def layer(x, gain, wgu, wd, att, stream=None):
    from paper_2510_11331_amd import add_rmsnorm_q, gate_up_q, linear_q
    x, q, e = add_rmsnorm_q(x, gain, 1e-5, add=att, stream=stream)
    q, e = gate_up_q(q, e, wgu, stream=stream)
    return linear_q(q, e, wd, add=x, stream=stream)


def layer_inputs(M, d, F, seed):
    import torch
    from paper_2510_11331_amd import pack_linear_q
    from paper_2510_11331_amd.engine import interleave_gate_up
    r = np.random.default_rng(seed)
    gate, up, down = (0.02 * r.normal(size=s).astype(np.float32) for s in ((F, d), (F, d), (d, F)))
    x, att = r.normal(size=(M, d)).astype(np.float32), 0.3 * r.normal(size=(2, M, d)).astype(np.float32)
    gain = (1 + 0.1 * r.normal(size=d)).astype(np.float32)
    w = [t(interleave_gate_up(gate, up)), t(down)]
    return t(x), t(gain, torch.bfloat16), pack_linear_q(w[0]), pack_linear_q(w[1]), t(att), (w[0], w[1])


@pytest.mark.parametrize("M,d,F", [(1, 320, 448), (40, 768, 1040), (130, 512, 1408)])
def test_layer(M, d, F):
    """A layer's feed-forward pass against float64 with codes at the same three places; then against no codes at all: each
    code is within 2^-4 of its value, independently, so a sum of products of two is about sqrt(2) 2^-4 / sqrt(3) (a uniform
    error) of its root mean square off, gate and up both, and the down product again: 0.15 is over twice that."""
    say("layer", M, d, F)
    x, gain, wgu, wd, att, (w1, w2) = layer_inputs(M, d, F, M)
    got = host(layer(x, gain, wgu, wd, att)) - (s := (host(x) + host(att).sum(0)))
    s32 = s.astype(np.float32).astype(np.float64)
    y = qref.norm(s32, host(gain)[None], 1e-5)
    h = qref.row_values(*qref.quantise_rows(y.astype(np.float32).astype(np.float64)), d) @ qref.weight_values(*qref.quantise_weight(host(w1))).T
    h = qref.swiglu(h)
    want = qref.row_values(*qref.quantise_rows(h), F) @ qref.weight_values(*qref.quantise_weight(host(w2))).T
    # of F codes, a share 2^4 CUT8 may fall on the other side of a rounding: steps of 2^-3 of as many terms
    assert np.linalg.norm(got - want) <= (2.0 ** -3 * math.sqrt(16 * CUT8) + 1e-5) * np.linalg.norm(want)
    plain = qref.swiglu(y @ host(w1).T) @ host(w2).T
    assert np.linalg.norm(got - plain) <= 0.15 * np.linalg.norm(plain)


def test_streams_and_graphs():
    """Calls on two streams at once, each with its own rows; a captured pass replayed between eager ones and beside a second
    captured one; every result equal to the eager call's, bit for bit."""
    import torch
    say("streams and graphs")
    sets = [layer_inputs(M, 512, 1040, 20 + M)[:5] for M in (5, 150)]
    want = [layer(*a) for a in sets]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in st:
        s.wait_stream(torch.cuda.current_stream())
    got = [[layer(*a, stream=s) for a, s in zip(sets, st)] for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for gs in got for g, w in zip(gs, want))
    graphs, outs = [], []
    for a in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(layer(*a))
        graphs.append(g)
    for n in range(4):
        for o in outs:
            o.zero_()
        if n % 2:                                              # both at once
            for s in st:
                s.wait_stream(torch.cuda.current_stream())
            for g, s in zip(graphs, st):
                with torch.cuda.stream(s):
                    g.replay()
        else:
            for g in graphs:
                g.replay()
        eager = [layer(*a) for a in sets]
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(outs + eager, want + want))


# ------------------------------------------------------------------ ranges, tiles, borders


# few rows: K in 4 ranges with one tile a workgroup, 2 ranges, 4 and 2 ranges with two tiles, four tiles a workgroup whose
# runs cross a block of 128 rows; more rows: row tiles with and without ranges, as the planner picks them (every one of them, by
# name: test_gpu_ffn_q_sums.py); K past the streamed scales
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(3, 500, 10300), (64, 1000, 2560), (64, 1500, 5200), (50, 3000, 5130), (20, 16130, 140), (64, 4200, 300),
                                   (70, 300, 10000), (65, 300, 4200), (200, 2100, 8400), (200, 8200, 140), (769, 5000, 140), (65, 4100, 8400),
                                   (769, 2100, 1500), (65, 8200, 8400), (3, 40, 16500), (64, 33, 40000), (1200, 300, 700), (4000, 130, 2200),
                                   (65, 8200, 11000), (65, 12000, 6000), (4200, 130, 6000), (2100, 130, 8400), (2100, 520, 11000),
                                   (1000, 8200, 140), (100, 5000, 6000), (400, 8200, 14000)])
def test_linear_ranges_and_tiles(M, N, K, dtype):
    import torch
    from paper_2510_11331_amd import linear_q
    say("linear ranges", M, N, K, dtype)
    r = np.random.default_rng([M, N, K])
    c, E, q, e = rows8(r, M, K)
    wc, wE, w = weight8(r, N, K)
    a, b = torch.from_numpy(qref.row_values(c, E, K)), torch.from_numpy(qref.weight_values(wc, wE))
    add = r.normal(size=(M, N)).astype(np.float32)
    want, mag = (a @ b.T).numpy() + add, (a.abs() @ b.abs().T).numpy() + np.abs(add)
    check_product(host(linear_q(q, e, w, add=t(add), dtype=dt(dtype))), want, mag, K, dtype)


@pytest.mark.parametrize("M,F,K", [(3, 6000, 140), (20, 10000, 260), (33, 14000, 130), (64, 18000, 130), (64, 16400, 20), (3, 48, 16500), (65, 288, 140),
                                   (2050, 992, 140), (769, 4992, 140), (769, 8192, 140),
                                   (130, 12016, 1000), (400, 12016, 270)])
def test_gate_up_tiles(M, F, K):
    """Few rows: 4, 6 and 8 tiles a workgroup, more than one round of them; K past the streamed scales; every row tile."""
    import torch
    from paper_2510_11331_amd import gate_up_q
    say("gate_up tiles", M, F, K)
    r = np.random.default_rng([M, F, K])
    c, E, q, e = rows8(r, M, K, 0.5)
    wc, wE, w = weight8(r, 2 * F, K)
    a, b = torch.from_numpy(qref.row_values(c, E, K)), torch.from_numpy(qref.weight_values(wc, wE))
    mag = (a.abs() @ b.abs().T).numpy()
    tol = sum_error(K, mag) + (CUT8 * mag if M > 64 or K > 16384 else 0)
    p = (a @ b.T).numpy()
    check_codes_of(*gate_up_q(q, e, w), qref.swiglu(p), swiglu_error(p, tol))


@pytest.mark.parametrize("M", [5, 40, 300])
def test_only_its_own_memory(M):
    """Every buffer ends in bytes that no call may touch: codes, exponents, outputs, workspaces, x_out; rows of the input
    behind the last are not read (NaN codes)."""
    import torch
    from paper_2510_11331_amd import _lib
    say("own memory", M)
    L, F32 = _lib.lib(), _lib.SD_DTYPE_F32
    r = np.random.default_rng(M)
    d, F = 700, 10320
    s = torch.cuda.current_stream().cuda_stream
    made = []

    def buf(n, fill=0x7f):
        b = torch.full((n + 512,), fill, dtype=torch.uint8, device="cuda")
        made.append((b, n, fill))
        return b

    x, add, gain = (t(r.normal(size=k).astype(np.float32)) for k in ((M, d), (2, M, d), (d,)))
    w1, w2 = (t((0.02 * r.normal(size=k)).astype(np.float32)) for k in ((2 * F, d), (d, F)))
    p1, p2 = buf(L.sd_linear_q_bytes(2 * F, d)), buf(L.sd_linear_q_bytes(d, F))
    xo, q, e, h, eh, out = buf(M * d * 4), buf(M * 768), buf(M * 8), buf(M * 10368), buf(M * 84), buf(M * d * 4)
    n1, n2 = L.sd_gate_up_q_workspace_bytes(M, F, d), L.sd_linear_q_workspace_bytes(M, d, F)
    assert n2 or M == 300
    ws1, ws2 = buf(n1), buf(n2)
    P = lambda b: b.data_ptr()
    assert L.sd_pack_linear_q(P(w1), P(p1), 2 * F, d, F32, s) == L.sd_pack_linear_q(P(w2), P(p2), d, F, F32, s) == 0
    assert L.sd_add_rmsnorm_q(M, d, F32, P(x), 2, P(add), P(xo), P(gain), F32, 1e-5, P(q), P(e), s) == 0
    assert L.sd_gate_up_q(M, F, d, P(q), P(e), P(p1), P(h), P(eh), P(ws1), n1, s) == 0
    assert L.sd_linear_q(M, d, F, P(h), P(eh), P(p2), P(xo), P(out), d, F32, P(ws2), n2, s) == 0
    torch.cuda.synchronize()
    assert all(bool((b[n:] == fill).all()) for b, n, fill in made)
    y = out[:M * d * 4].view(torch.float32)
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("M", [3, 100])
def test_scale_of_nan(M):
    """E = 255 of a row's block or of a weight's block makes NaN of the sums that it enters and of no others."""
    import torch
    from paper_2510_11331_amd import LinearQ, linear_q
    say("nan scale", M)
    r = np.random.default_rng(13)
    N, K = 300, 700
    c, E, q, _ = rows8(r, M, K)
    wc, wE, w = weight8(r, N, K)
    E, wE2 = E.copy(), wE.copy()
    E[1, 2] = 255
    wE2[1, 3] = 255
    e, w2 = t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu), LinearQ(t(qref.pack(wc, wE2)), N, K)
    for dtype in ("fp32", "bf16"):
        nan = np.isnan(host(linear_q(q, e, w, dtype=dt(dtype))))
        assert nan[1].all() and nan.sum() == N
        nan = np.isnan(host(linear_q(q, e, w2, dtype=dt(dtype))))
        assert nan[1].all() and nan[:, 128:256].all() and nan.sum() == N + 128 * (M - 1)


@pytest.mark.parametrize("M", [3, 100])
def test_gate_up_nan_row(M):
    """A row of NaN: F codes of NaN, padding zero; the other rows as without it."""
    import torch
    from paper_2510_11331_amd import gate_up_q
    say("gate_up nan row", M)
    r = np.random.default_rng(14)
    F, K = 272, 300
    c, E, q, e = rows8(r, M, K, 0.5)
    _, _, w = weight8(r, 2 * F, K)
    want = [host(a) for a in gate_up_q(q, e, w)]
    c = c.copy()
    c[1, 299] = 0x7f
    got = [host(a) for a in gate_up_q(t(c).view(torch.float8_e4m3fn), e, w)]
    assert (got[0][1, :F] & 127 == 127).all() and not got[0][1, F:].any()
    rest = [i for i in range(M) if i != 1]
    assert all(np.array_equal(g[rest], v[rest]) for g, v in zip(got, want))


def test_packed_past_32_bits():
    """A packed matrix of more than 2^32 bytes: tiles of its start, middle and end, and a product with it."""
    import torch
    from paper_2510_11331_amd import linear_q, pack_linear_q
    say("pack large")
    N, K, n = 65600, 66000, 1312                              # rows and columns repeat: N = 50 n, K = 500 x 132
    r = np.random.default_rng(15)
    small = t((0.02 * r.normal(size=(n, 132))).astype(np.float32), torch.bfloat16)
    w = pack_linear_q(small.repeat(50, 500))
    assert w.codes.numel() > 1 << 32
    kb = 516
    tiles = w.codes.view(torch.uint8).view(N // 16, kb, 2048)
    full = small.double().cpu().numpy()
    for row0 in (0, 32768, 65536 - 128):
        block = np.take(np.tile(full, (1, 10)), np.arange(row0, row0 + 128) % n, axis=0)
        for b in (0, 258, 514):
            cols = np.take(block, np.arange(128 * b, 128 * b + 128) % 132, axis=1)
            data = qref.pack(*qref.quantise_weight(cols))
            assert np.array_equal(tiles[row0 // 16:row0 // 16 + 8, b].reshape(-1).cpu().numpy(), data[:128 * 128])
            assert int(host(w.exps)[row0 // 128, b]) == data[128 * 128]
    K2 = 66000                                                # rows that pick one column each, of every eighth part of K
    pick = np.zeros((8, K2))
    at = [8250 * i + 7 * i for i in range(8)]
    pick[np.arange(8), at] = 1.0
    c, E = qref.quantise_rows(pick)
    got = host(linear_q(t(c).view(torch.float8_e4m3fn), t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu), w))
    for i, k in enumerate(at):
        for row0 in (0, 32768, 65536 - 128):
            rows, cols = np.arange(row0, row0 + 128) % n, np.arange(k // 128 * 128, k // 128 * 128 + 128) % 132
            block = full[np.ix_(rows, cols)]
            v = qref.weight_values(*qref.quantise_weight(block))[:, k % 128]
            assert np.allclose(got[i, row0:row0 + 128], v, rtol=4 * U32, atol=0)


def test_ranges_in_graphs():
    """Products with K ranges, captured twice (each with the workspace of its capture), replayed at once on two streams
    between eager ones: bit for bit the eager results."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("ranges in graphs")
    r = np.random.default_rng(16)
    sets = []
    for M, N, K in ((40, 700, 10300), (70, 300, 10000)):
        _, _, q, e = rows8(r, M, K)
        sets.append((q, e, weight8(r, N, K)[2]))
    want = [linear_q(*a) for a in sets]
    torch.cuda.synchronize()
    st, graphs, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for a in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(linear_q(*a))
        graphs.append(g)
    for _ in range(4):
        for o in outs:
            o.zero_()
        for s in st:
            s.wait_stream(torch.cuda.current_stream())
        for g, s in zip(graphs, st):
            with torch.cuda.stream(s):
                g.replay()
        eager = [linear_q(*a) for a in sets]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs + eager, want + want))
