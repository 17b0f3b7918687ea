"""The 8-bit products' sums against float64, with bounds that one lost block or one lost bit would break (qsums)."""
import numpy as np
import pytest

import qplans
import qref
import qsums
import test_gpu_ffn_q as plain
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


def check_codes(got, product, err):
    """The rows that gate_up_q returned for a product known to err."""
    h, err = qref.swiglu(product), qsums.swiglu_error(product, err)
    q, exps = (host(x) for x in got)
    F, blocks = h.shape[1], -(-h.shape[1] // 128)
    E = exps[:, :blocks].astype(np.int64)
    assert not q[:, F:].any() and not exps[:, blocks:].any()
    hc, hE = qref.quantise_rows(h)
    scale = np.repeat(2.0 ** (np.maximum(E, hE) - 127.0), 128, 1)[:, :F]
    assert qsums.codes_ok(qref.row_values(q, E, F), h, err, qref.row_values(hc, hE, F), scale)


def check_gate_up(M, F, K, fast=False):
    from paper_2510_11331_amd import gate_up_q
    a, w, q, e, wq = operands(M, 2 * F, K, 0.5)
    p, s = qsums.terms(a, w)
    check_codes(gate_up_q(q, e, wq, fast=fast), p, qsums.sum_error(K, s))


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


# ------------------------------------------------------------------ every plan


def codes8(M, N, K, n_exp, w_exp):
    """Random codes and a scale of its own for every block: values [M, K] and [N, K] in float64, and what the calls take, made
    on the GPU.  n_exp, w_exp: ranges of the scales' exponents."""
    import torch
    from paper_2510_11331_amd import LinearQ
    g = torch.Generator(device="cuda")
    g.manual_seed(M * 1000003 + N * 1009 + K)

    def operand(R, R16, lo_hi, E_rows):
        v = torch.zeros(R16, qref.up(K, 128), device="cuda")
        v[:R, :K] = (60 * torch.randn(R, K, generator=g, device="cuda")).clamp(-448, 448)
        v = v.to(torch.float8_e4m3fn)
        E = torch.randint(*lo_hi, (E_rows, v.shape[1] // 128), generator=g, device="cuda")
        exps = torch.zeros(E_rows, qref.up(E.shape[1], 4), dtype=torch.uint8, device="cuda")
        exps[:, :E.shape[1]] = E
        return v, E, exps

    q, E, e = operand(M, M, n_exp, M)
    v, F, f = operand(N, qref.up(N, 16), w_exp, -(-N // 128))
    tiles = v.view(torch.uint8).view(v.shape[0] // 16, 16, -1, 2, 4, 16).permute(0, 2, 3, 4, 1, 5)
    w = LinearQ(torch.cat([tiles.reshape(-1), f.reshape(-1)]), N, K)
    scale = lambda E, n: torch.ldexp(torch.ones_like(E, dtype=torch.float64), E - 127).repeat_interleave(n, 0)
    a = q.double().view(M, -1, 128) * scale(E, 1)[..., None]
    b = v.double().view(v.shape[0], -1, 128) * scale(F, 128)[:v.shape[0], :, None]
    return a.view(M, -1)[:, :K], b.view(v.shape[0], -1)[:N, :K], q, e.view(torch.float8_e8m0fnu), w


def terms_gpu(a, b):
    return host(a @ b.t().contiguous()), host(((a * a) @ (b * b).t().contiguous()).sqrt())


@pytest.mark.parametrize("fast,rows,cols,ranges,M,N,K", qplans.LINEAR)
def test_linear_plan(fast, rows, cols, ranges, M, N, K):
    """Every kernel and number of K ranges, past the start of its loop, for both types, with an addend of the sum's size."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("linear plan", fast, rows, cols, ranges, M, N, K)
    assert qplans.plan("linear", M, N, K, fast) == qplans.expected(fast, rows, cols, ranges, M)
    a, b, q, e, w = codes8(M, N, K, (117, 121), (115, 120))
    want, s = terms_gpu(a, b)
    err = qsums.cut_error(s) if fast else qsums.sum_error(K, s)
    for dtype in ("fp32", "bf16"):
        assert qsums.product_ok(host(linear_q(q, e, w, dtype=dt(dtype), fast=bool(fast))), want, err, dtype)
    add = torch.randn(M, N, device="cuda")
    got = host(linear_q(q, e, w, add=add, fast=bool(fast)))
    assert qsums.product_ok(got, want + host(add), err + 2 * qsums.STEP32 * np.abs(host(add)), "fp32")


@pytest.mark.parametrize("fast,rows,cols,ranges,M,F,K", qplans.GATE_UP)
def test_gate_up_plan(fast, rows, cols, ranges, M, F, K):
    from paper_2510_11331_amd import gate_up_q
    say("gate_up plan", fast, rows, cols, M, F, K)
    assert qplans.plan("gate_up", M, F, K, fast) == qplans.expected(fast, rows, cols, ranges, M)
    a, b, q, e, w = codes8(M, 2 * F, K, (117, 121), (115, 120))
    p, s = terms_gpu(a, b)
    err = qsums.cut_error(s) if fast else qsums.sum_error(K, s)
    check_codes(gate_up_q(q, e, w, fast=bool(fast)), p, err)


# ------------------------------------------------------------------ extreme scales


@pytest.mark.parametrize("fast", [False, True])
@pytest.mark.parametrize("M", [6, 100])
def test_extreme_scales(M, fast):
    """Rows whose blocks have scales of 2^-126 to 2^127, with nonzero codes in every block, and a weight with a large and
    a small block of its own: the product of two blocks' scales is held within 2^-126 (a smaller one counts as zero) and 2^127."""
    import torch
    from paper_2510_11331_amd import LinearQ, linear_q
    say("extreme scales", M, fast)
    r = np.random.default_rng(M)
    N, K = 300, 500
    c, E = qref.quantise_rows(r.normal(size=(M, K)))
    wc, wF = qref.quantise_weight(r.normal(size=(N, K)))
    tiny = lambda shape: np.where(r.integers(0, 2, size=shape) == 1, 0x81, 0x01).astype(np.uint8)     # +- 2^-9
    E, wF = E.copy(), wF.copy()
    wF[:] = 118
    wF[1], wF[2] = 140, 1                                      # rows 128 to 255 and 256 to 299 of the weight
    wc[128:256] = tiny((128, K))
    E[:] = 127
    E[0] = 1                                                   # far below 2^-126
    E[1] = 10                                                  # 10 + 118 - 254 = -126: the smallest that counts
    E[2] = 9                                                   # the largest that does not
    E[3] = 254                                                 # 254 + 140 - 254 = 140: held at 2^127
    E[4] = [1, 10, 100, 120]                                   # beside each other
    c[3] = np.where(np.arange(c.shape[1]) < K, tiny(c.shape[1]), 0)
    e = E[:, :, None].astype(np.int64) + np.repeat(wF, 128, 0)[:N].T[None] - 254                      # [M, blocks, N]
    if not fast or M <= 64:
        e = np.where(e < -126, -5000, np.minimum(e, 127))
    pad = lambda v: np.pad(v, ((0, 0), (0, 512 - K))).reshape(len(v), 4, 128)
    a, b = pad(qref.value(c)[:, :K]), pad(qref.value(wc))
    s = np.stack([a[:, k] @ b[:, k].T for k in range(4)], 1)                                          # [M, blocks, N]
    root = np.stack([np.sqrt((a[:, k] ** 2) @ (b[:, k] ** 2).T) for k in range(4)], 1)
    want, root = np.ldexp(s, e).sum(1), np.sqrt((np.ldexp(root, e) ** 2).sum(1))
    # the 8-bit instruction takes the scales as they are: with 2^140 partial sums pass fp32's largest number, and may be infinite
    over = 8 * root > 2.0 ** 128
    assert not over[:3].any() and (fast and M > 64 or not over.any())
    q, ex = t(c).view(torch.float8_e4m3fn), t(qref.exps_bytes(E)).view(torch.float8_e8m0fnu)
    got = host(linear_q(q, ex, LinearQ(t(qref.pack(wc, wF)), N, K), fast=fast))
    err = (qsums.cut_error(root) if fast and M > 64 else qsums.sum_error(K, root)) + 2.0 ** -149
    got, want = np.where(over, 0, got), np.where(over, 0, want)
    for i in range(M):                                         # each row is of a size of its own
        for part in (slice(0, 128), slice(128, 256), slice(256, N)):
            assert np.linalg.norm(got[i, part] - want[i, part]) <= np.linalg.norm(err[i, part]), (i, part)


# ------------------------------------------------------------------ the caller's choice


@pytest.mark.parametrize("M", [64, 300])
def test_fast_on_streams_and_in_graphs(M):
    """fast goes along to another stream and into a graph, with K in ranges and without; up to 64 rows it changes nothing, above
    it is another result; each replay is the eager call's, bit for bit."""
    import torch
    from paper_2510_11331_amd import gate_up_q, linear_q
    say("fast on streams", M)
    gu, down = codes8(M, 2 * 528, 1110, (117, 121), (115, 120))[2:], codes8(M, 520, 6000, (117, 121), (115, 120))[2:]
    assert M == 64 or qplans.plan("linear", M, 520, 6000, 1)[4] > 1

    def both(fast, stream=None):
        return [x.view(torch.uint8) if x.element_size() == 1 else x
                for x in (*gate_up_q(*gu, stream=stream, fast=fast), linear_q(*down, stream=stream, fast=fast),
                          linear_q(*down, dtype=torch.bfloat16, stream=stream, fast=fast))]

    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    exact, want = both(False), both(True)
    assert same(exact, want) == (M <= 64)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    got = both(True, other)
    torch.cuda.synchronize()
    assert same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(True)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
        eager = both(True), both(False)
        torch.cuda.synchronize()
        assert same(outs, want) and same(eager[0], want) and same(eager[1], exact)


@pytest.fixture
def all_fast(monkeypatch):
    """The public calls with fast=True, and the library's fast calls in the place of the others."""
    import functools
    import paper_2510_11331_amd as P
    monkeypatch.setattr(P, "linear_q", functools.partial(P.linear_q, fast=True))
    monkeypatch.setattr(P, "gate_up_q", functools.partial(P.gate_up_q, fast=True))
    from paper_2510_11331_amd import _lib
    L = _lib.lib()
    for name in ("sd_linear_q", "sd_gate_up_q"):
        monkeypatch.setattr(L, name, getattr(L, name + "_fast"))


@pytest.mark.parametrize("name,args", [
    ("test_linear", (65, 144, 384, "bf16")), ("test_linear", (257, 129, 1100, "bf16")), ("test_linear_add_and_strides", (200, "bf16")),
    ("test_linear_offsets_past_32_bits", ()), ("test_gate_up", (130, 272, 700)), ("test_gate_up", (300, 1040, 260)), ("test_layer", (130, 512, 1408)),
    ("test_streams_and_graphs", ()), ("test_only_its_own_memory", (300,)), ("test_scale_of_nan", (100,)), ("test_gate_up_nan_row", (100,)),
    ("test_ranges_in_graphs", ())])
def test_fast_borders(all_fast, name, args):
    """The plain calls' tests of strides, untouched memory, NaN, offsets past 32 bits and graphs, of the fast ones (fp32 outputs are
    bounded in test_linear_plan)."""
    getattr(plain, name)(*args)


def test_fast_nan_code(all_fast):
    """A NaN code makes NaN of its row's outputs and no others."""
    import torch
    from paper_2510_11331_amd import linear_q
    say("fast, a NaN code")
    _, _, q, e, w = codes8(100, 300, 700, (117, 121), (115, 120))
    q.view(torch.uint8)[7, 650] = 0xff
    for dtype in (torch.float32, torch.bfloat16):
        nan = np.isnan(host(linear_q(q, e, w, dtype=dtype)))
        assert nan[7].all() and nan.sum() == 300
