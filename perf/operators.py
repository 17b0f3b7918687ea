"""Performance cases of the feed-forward network in 8-bit floating point: the
operators of paper_2510_11331_amd.ffn_q, called as a serving program calls them.

A case is a dict of plain values with a "kind":

  pack     a weight matrix is quantised and laid out (once, when a model is loaded)
  norm     residual addition, RMSNorm and the 8-bit output of one pass's rows
  linear   the product of 8-bit rows with a packed weight (the down projection)
  gate_up  the gate/up product with SwiGLU and its 8-bit output

Numbers in 8 bits are e4m3 codes with one scale 2^(E - 127) per 128 entries of an
activation row and per 128 x 128 block of a weight; E is the smallest E >= 1 with
max |v| <= 448 2^(E - 127).  Sizes are those of the repository's model pairs (7B:
width 4096, feed-forward 11008; 13B: 5120, 13824; small target: 2048, 5632; drafts:
1024, 2816) at one row (a single token), at the rows of batched verification
(tasks x (speculation length + 1)) and at those of prefill chunks, and odd ones.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
BLOCK = 128
EPS = 1e-5


def listed():
    return [
        # loading a draft model's down projection
        dict(name="pack_draft_down", kind="pack", n=1024, k=2816, dtype="bf16"),
        # loading the gate/up projection of a 7B layer
        dict(name="pack_7b_gate_up", kind="pack", n=22016, k=4096, dtype="bf16"),
        # a single token's row in the 7B model: latency
        dict(name="norm_7b_row", kind="norm", rows=1, d=4096, adds=0, dtype="fp32"),
        # verification of 8 tasks, after an O projection in four K ranges
        dict(name="norm_7b_b8", kind="norm", rows=40, d=4096, adds=4, dtype="fp32"),
        # a prefill chunk of the 13B model, residual stream in 16 bits
        dict(name="norm_13b_prefill", kind="norm", rows=2048, d=5120, adds=1, dtype="bf16"),
        # one token through an odd-sized projection: the smallest call
        dict(name="linear_odd_row", kind="linear", rows=1, n=1000, k=1000, dtype="fp32", add=False),
        # down projection of the 7B verification pass at 8 tasks
        dict(name="down_7b_b8", kind="linear", rows=40, n=4096, k=11008, dtype="fp32", add=False),
        # down projection of the 13B verification pass at 64 tasks, added to the residual stream
        dict(name="down_13b_b64", kind="linear", rows=320, n=5120, k=13824, dtype="fp32", add=True),
        # down projection of a 7B prefill chunk
        dict(name="down_7b_prefill", kind="linear", rows=2048, n=4096, k=11008, dtype="bf16", add=False),
        # gate/up of the small target, verification of one task at speculation length 4
        dict(name="gate_up_small_b1", kind="gate_up", rows=5, f=5632, k=2048),
        # gate/up of the 7B verification pass at 8 tasks: what dominates the step
        dict(name="gate_up_7b_b8", kind="gate_up", rows=40, f=11008, k=4096),
        # gate/up of a 7B prefill chunk
        dict(name="gate_up_7b_prefill", kind="gate_up", rows=2048, f=11008, k=4096),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["pack", "norm", "norm", "linear", "linear", "linear", "gate_up", "gate_up"])
    if kind == "pack":
        return dict(kind=kind, n=_log_uniform(rng, 64, 22016), k=_log_uniform(rng, 64, 4096),
                    dtype=rng.choice(["bf16", "fp32"]))
    rows = _log_uniform(rng, 1, 2048)
    if kind == "norm":
        return dict(kind=kind, rows=rows, d=_log_uniform(rng, 64, 5120), adds=rng.randint(0, 4 if rows < 512 else 1),
                    dtype=rng.choice(["bf16", "fp32"]))
    if kind == "linear":
        return dict(kind=kind, rows=rows, n=_log_uniform(rng, 64, 5120), k=_log_uniform(rng, 64, 13824),
                    dtype=rng.choice(["bf16", "fp32"]), add=rng.random() < 0.4)
    return dict(kind=kind, rows=rows, f=16 * _log_uniform(rng, 8, 688), k=_log_uniform(rng, 64, 4096))


# --------------------------------------------------------------------------
# the format, in elementary operations


def _up(n, m):
    return -(-n // m) * m


def _exponents(amax):
    """E of blocks with the maxima amax (float32 or float64), as int32."""
    m, e = torch.frexp(amax)                              # amax = m 2^e, m in [0.5, 1); 448 = 0.875 2^9
    E = e.to(torch.int32) + (m > 0.875).to(torch.int32) + (127 - 9)
    return torch.where(amax > 0, E.clamp(min=1), torch.ones_like(E))


def _power(E):
    """2^(E - 127) as float32, 1 <= E <= 254."""
    return (E << 23).view(torch.float32)


def _quantise_rows(y):
    """y [M, K] float32 -> codes [M, K padded to 128] float8_e4m3fn, E [M, blocks] int32."""
    M, K = y.shape
    v = torch.nn.functional.pad(y, (0, _up(K, BLOCK) - K)).view(M, -1, BLOCK)
    E = _exponents(v.abs().amax(-1))
    return (v * _power(254 - E)[..., None]).view(M, -1).to(torch.float8_e4m3fn), E


def _exps_bytes(E):
    """E [M, blocks] -> float8_e8m0fnu [M, blocks padded to 4 with zero bytes]."""
    b = E.to(torch.uint8)
    return torch.nn.functional.pad(b, (0, _up(b.shape[1], 4) - b.shape[1])).view(torch.float8_e8m0fnu)


def _quantise_weight(w):
    """w [N, K] -> codes [N, K] float8_e4m3fn, E [N / 128, K / 128] int32 (both rounded up)."""
    N, K = w.shape
    v = torch.nn.functional.pad(w.float(), (0, _up(K, BLOCK) - K, 0, _up(N, BLOCK) - N))
    v = v.view(-1, BLOCK, _up(K, BLOCK) // BLOCK, BLOCK)
    E = _exponents(v.abs().amax((1, 3)))
    q = (v * _power(254 - E)[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(_up(N, BLOCK), _up(K, BLOCK)).view(torch.uint8)[:N, :K].contiguous().view(torch.float8_e4m3fn), E


def _pack(codes, E):
    """The packed layout: 2 KB tiles of 16 rows x 128 columns, row tiles major, as
    [64-byte half][16-byte unit][row][16 bytes]; then E row by row, padded to 4 bytes."""
    N, K = codes.shape
    b = torch.nn.functional.pad(codes.view(torch.uint8), (0, _up(K, BLOCK) - K, 0, _up(N, 16) - N))
    tiles = b.view(_up(N, 16) // 16, 16, _up(K, BLOCK) // BLOCK, 2, 4, 16).permute(0, 2, 3, 4, 1, 5).reshape(-1)
    return tiles.view(torch.float8_e4m3fn), _exps_bytes(E)


def _row_values(codes, exps, K):
    M = codes.shape[0]
    blocks = codes.shape[1] // BLOCK
    scale = _power(exps.view(torch.uint8)[:, :blocks].to(torch.int32))
    return (codes.float().view(M, blocks, BLOCK) * scale[..., None]).view(M, -1)[:, :K]


def _weight_values(codes, E):
    N, K = codes.shape
    scale = _power(E).repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return codes.float() * scale


# --------------------------------------------------------------------------
# inputs


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(g, rows, k):
    """Rows as a norm or a SwiGLU leaves them: of different sizes, with a few large channels."""
    size = torch.exp(0.5 * _randn(g, rows, 1))
    channel = torch.exp(0.7 * _randn(g, 1, k))
    return _quantise_rows(_randn(g, rows, k) * size * channel)


def _weight(g, n, k):
    return 0.02 * _randn(g, n, k)


def _packed(codes, E):
    tiles, exps = _pack(codes, E)
    return torch.cat([tiles.view(torch.uint8), exps.view(torch.uint8).reshape(-1)])


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "pack":
        s["w"] = _weight(g, case["n"], case["k"]).to(_type(case))
    elif kind == "norm":
        M, d, t = case["rows"], case["d"], _type(case)
        s["x"] = _randn(g, M, d).to(t)
        s["add"] = (0.3 * _randn(g, case["adds"], M, d)).to(t) if case["adds"] else None
        s["gain"] = (1.0 + 0.1 * _randn(g, d)).to(torch.bfloat16)
    else:
        rows, k = case["rows"], case["k"]
        n = case["n"] if kind == "linear" else 2 * case["f"]
        q, E = _rows(g, rows, k)
        s["q"], s["exps"] = q, _exps_bytes(E)
        s["codes"], s["E"] = _quantise_weight(_weight(g, n, k))
        s["packed"] = _packed(s["codes"], s["E"])
        if kind == "linear":
            s["add"] = _randn(g, rows, n) if case["add"] else None
    return s


# --------------------------------------------------------------------------
# one pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2510_11331_amd import ffn_q
        if kind == "pack":
            wq = ffn_q.pack_linear_q(s["w"])
            return {"codes": wq.codes, "exps": wq.exps}
        if kind == "norm":
            x, q, exps = ffn_q.add_rmsnorm_q(s["x"], s["gain"], EPS, add=s["add"])
            return {"x": x, "q": q, "exps": exps}
        if kind == "linear":
            wq = ffn_q.LinearQ(s["packed"], case["n"], case["k"])
            return {"out": ffn_q.linear_q(s["q"], s["exps"], wq, add=s["add"], dtype=_type(case))}
        wq = ffn_q.LinearQ(s["packed"], 2 * case["f"], case["k"])
        q, exps = ffn_q.gate_up_q(s["q"], s["exps"], wq)
        return {"q": q, "exps": exps}
    if kind == "pack":
        codes, exps = _pack(*_quantise_weight(s["w"]))
        return {"codes": codes, "exps": exps}
    if kind == "norm":
        # in 64 bits: the sum is rounded once, to the stored type, and the normed value to a code
        x = s["x"]
        if s["add"] is not None:
            x = torch.cat([x[None].double(), s["add"].double()]).sum(0).to(x.dtype)
        v = x.double()
        y = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * s["gain"].double()
        q, E = _quantise_rows(y.float())
        return {"x": x, "q": q, "exps": _exps_bytes(E)}
    out = _row_values(s["q"], s["exps"], case["k"]) @ _weight_values(s["codes"], s["E"]).t()
    if kind == "linear":
        if s["add"] is not None:
            out = s["add"] + out
        return {"out": out.to(_type(case))}
    gate_up = out.view(case["rows"], -1, 2, 16)           # 16 gate rows, then their 16 up rows
    gate, up = gate_up[:, :, 0].reshape(case["rows"], -1), gate_up[:, :, 1].reshape(case["rows"], -1)
    q, E = _quantise_rows(gate / (1.0 + torch.exp(-gate)) * up)
    return {"q": q, "exps": _exps_bytes(E)}


# --------------------------------------------------------------------------
# what a pass cannot do without


def work(case):
    kind = case["kind"]
    size = 2.0 if case.get("dtype") == "bf16" else 4.0
    if kind == "pack":
        values = float(case["n"]) * case["k"]
        return dict(bytes=values * (size + 1), flops=2 * values)
    if kind == "norm":
        values = float(case["rows"]) * case["d"]
        reads = 1 + case["adds"] + (1 if case["adds"] else 0)
        return dict(bytes=values * (size * reads + 1 + 1 / BLOCK) + 2.0 * case["d"], flops=values * (5 + case["adds"]))
    rows, k = float(case["rows"]), float(case["k"])
    if kind == "linear":
        n = float(case["n"])
        return dict(bytes=(rows + n) * k + rows * n * (size + (4 if case["add"] else 0)), flops=2 * rows * n * k)
    f = float(case["f"])
    return dict(bytes=(rows + 2 * f) * k + rows * f * (1 + 1 / BLOCK), flops=4 * rows * f * k)


# --------------------------------------------------------------------------
# from the definition, in 64 bits


def _two(e):
    """2^e for whole numbers e, as float64 (its exponent field: pow is a last place off on some devices)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _code64(v):
    """Nearest e4m3 number (3 fraction bits, exponents from -6, ties to even) of float64 v, |v| <= 448."""
    _, e = torch.frexp(v)
    step = _two((e - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _scales64(v, dims):
    """2^(E - 127) of blocks: the smallest power of two, from 2^-126, times 448 that reaches the maximum."""
    a = v.abs().amax(dims, keepdim=True)
    s = _two(torch.ceil(torch.log2(a.clamp(min=1e-300) / 448.0)).clamp(min=-126.0))
    s = torch.where(a > 448.0 * s, 2.0 * s, s)            # the logarithm's own rounding
    return torch.where((a <= 224.0 * s) & (s > 2.0 ** -126), 0.5 * s, s)


def _split64(v, k):
    """[M, k] float64 -> zero-padded [M, blocks, 128]."""
    M = v.shape[0]
    out = torch.zeros(M, _up(k, BLOCK), dtype=torch.float64, device=v.device)
    out[:, :k] = v
    return out.view(M, -1, BLOCK)


def _rows64(y):
    """What a row operator returns for float64 y: codes and scales as numbers (2^-127 in the padding)."""
    v = _split64(y, y.shape[1])
    s = _scales64(v, (2,))
    exps = torch.full((y.shape[0], _up(v.shape[1], 4)), 2.0 ** -127, dtype=torch.float64, device=y.device)
    exps[:, :v.shape[1]] = s[..., 0]
    return _code64(v / s).view(y.shape[0], -1), exps


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "pack":
        w = s["w"].double()
        N, K = w.shape
        v = torch.zeros(_up(N, BLOCK), _up(K, BLOCK), dtype=torch.float64, device=w.device)
        v[:N, :K] = w
        v = v.view(-1, BLOCK, _up(K, BLOCK) // BLOCK, BLOCK)
        sc = _scales64(v, (1, 3))
        c = _code64(v / sc).reshape(-1, 16, _up(K, BLOCK) // BLOCK, 2, 4, 16)[:_up(N, 16) // 16]
        exps = torch.full((sc.shape[0], _up(sc.shape[2], 4)), 2.0 ** -127, dtype=torch.float64, device=w.device)
        exps[:, :sc.shape[2]] = sc[:, 0, :, 0]
        return {"codes": c.movedim(1, 4).reshape(-1), "exps": exps}
    if kind == "norm":
        x = s["x"].double()
        if s["add"] is not None:
            x = (x + s["add"].double().sum(0)).to(s["x"].dtype).double()      # as stored
        y = s["gain"].double() * x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / case["d"] + EPS)
        q, exps = _rows64(y.float().double())                                # codes are of the float32 value
        return {"x": x, "q": q, "exps": exps}
    k = case["k"]
    M = case["rows"]
    a = s["q"].double().view(M, -1, BLOCK)
    a = a * _two(s["exps"].view(torch.uint8).long()[:, :a.shape[1]] - 127)[..., None]
    a = a.view(M, -1)[:, :k].contiguous()
    N = s["codes"].shape[0]
    out = torch.empty(M, N, dtype=torch.float64, device=DEVICE)
    for n in range(0, N, BLOCK):
        w = s["codes"][n:n + BLOCK].double()
        w = w * _two(s["E"][n // BLOCK].long() - 127).repeat_interleave(BLOCK)[None, :k]
        out[:, n:n + BLOCK] = a @ w.t().contiguous()
    if kind == "linear":
        return {"out": out if s["add"] is None else out + s["add"].double()}
    rows = torch.arange(case["f"], device=DEVICE)
    gate = out[:, rows // 16 * 32 + rows % 16]
    up = out[:, rows // 16 * 32 + 16 + rows % 16]
    q, exps = _rows64(gate * torch.sigmoid(gate) * up)
    return {"q": q, "exps": exps}
