"""The 4-bit cache and its operators in float64 NumPy, from the definitions in include/sd.h: a code is found by
comparing against the table of all e2m1 numbers, a scale by trying powers of two."""
import numpy as np

POS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
U32 = 2.0 ** -24                                    # half a step of fp32, of bf16 2^-8, relative
HALF = {"bf16": 2.0 ** -8, "fp32": U32}


def code(v):
    """Nearest e2m1 codes of v, |v| <= 6 (ties to the even code)."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(POS, a), 1, 7)
    lo = hi - 1
    up = (POS[hi] - a < a - POS[lo]) | ((POS[hi] - a == a - POS[lo]) & (hi % 2 == 0))
    return (np.where(up, hi, lo) + np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def number(c):
    """e2m1 codes -> float64."""
    return np.where(c >= 8, -1.0, 1.0) * POS[c & 7]


def exponent(amax):
    """Smallest E >= 1 with amax <= 6 2^(E - 127)."""
    E = np.ones(amax.shape, dtype=np.int64)
    for k in range(2, 255):
        E = np.where(amax > 6.0 * 2.0 ** (k - 1 - 127), k, E)
    return E


def quantise(x):
    """[..., hd] -> codes [..., hd], E [..., hd / 32] (255: a NaN or an infinity among the 32)."""
    v = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    E = exponent(np.abs(v).max(-1))
    c = np.where(bad[..., None], 0, code(v * 2.0 ** (127.0 - E[..., None])))
    return c.reshape(x.shape).astype(np.uint8), np.where(bad, 255, E).astype(np.uint8)


def values(c, E):
    s = np.where(E == 255, np.nan, 2.0 ** (E.astype(np.float64) - 127.0))
    return number(c) * np.repeat(s, 32, -1)


class Pool:
    """The cache's bytes [blocks, KV, 17 hd]; `fill` in every byte that nothing writes."""

    def __init__(self, blocks, KV, hd, fill=0xff):
        self.KV, self.hd = KV, hd
        self.bytes = np.full((blocks, KV, 17 * hd), fill, dtype=np.uint8)
        t, j = np.arange(16)[:, None], np.arange(hd // 2)[None]     # byte j holds dimensions 2 j, 2 j + 1
        w = hd // 32                                                # bytes of a unit of hd / 16 dimensions
        self.kc = t * (hd // 2) + j
        self.vc = 8 * hd + ((t // 4 * 16 + j // w) * 4 + t % 4) * w + j % w
        b = np.arange(hd // 32)[None]
        self.ks = 16 * hd + t * (hd // 32) + b
        self.vs = 16 * hd + hd // 2 + b * 16 + t

    def put(self, page, t, k, v):
        """Keys and values [n, KV, hd] into tokens t [n] of pages [n]."""
        for x, at, scale in ((k, self.kc, self.ks), (v, self.vc, self.vs)):
            c, E = quantise(x)
            pair = c[..., 0::2] | c[..., 1::2] << 4
            for n in range(len(page)):
                self.bytes[page[n]][:, at[t[n]]] = pair[n]
                self.bytes[page[n]][:, scale[t[n]]] = E[n]

    def get(self, page, t):
        out = []
        for at, scale in ((self.kc, self.ks), (self.vc, self.vs)):
            x = np.empty((len(page), self.KV, self.hd))
            for n in range(len(page)):
                pair = self.bytes[page[n]][:, at[t[n]]]
                c = np.stack([pair & 15, pair >> 4], -1).reshape(self.KV, self.hd)
                x[n] = values(c, self.bytes[page[n]][:, scale[t[n]]])
            out.append(x)
        return out


def places(rows, lengths):
    """(sequence, position) of every row of sequences with so many rows and lengths."""
    b = np.repeat(np.arange(len(rows)), rows)
    pos = np.concatenate([np.arange(m - n, m) for n, m in zip(rows, lengths)] or [np.zeros(0, int)])
    return b, pos


def norm_rope(x, gain, cs, eps):
    """x [M, heads, hd], cs [M, hd / 2, 2] or None."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    if cs is not None:
        h = x.shape[-1] // 2
        a, b, c, s = x[..., :h], x[..., h:], cs[:, None, :, 0], cs[:, None, :, 1]
        x = np.concatenate([a * c - b * s, b * c + a * s], -1)
    return x


def attention(q, k, v, seen, scale):
    """q [n, H, hd], k and v [len, KV, hd], seen [n, len] -> (out, err): what the arithmetic may be off by before its
    rounding to the output's type, err[0] of fp32 and err[1] of bf16 outputs.

    A score is a sum of hd products, off by at most (hd + 4) steps (2 U32 each: the matrix unit may cut) of the sum of
    their magnitudes; a weight by e^(twice that), and by the rounding of the exponential's argument and result
    (8 + |score|) steps.  The weighted sum and the weights' sum are of at most n / 2 + 128 additions in a row.  A weight
    is held relative to the largest, which is 1, in fp32, whose normal numbers end at 2^-126: what is smaller may be
    lost, from the weight and from the parts it is split into (at most three).  It enters the product in 23 bits for
    fp32 outputs; for bf16 ones as two bf16 parts or as one fp16 number: 11 bits, a step's half being 2^-12 of it, and
    2^-25 below fp16's normal numbers."""
    n, H, hd = q.shape
    KV = k.shape[1]
    out, err = np.zeros((n, H, hd)), np.zeros((2, n, H, hd))
    if k.shape[0] == 0:
        return out, err
    count, some = seen.sum(1)[:, None], seen.any(1)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for h in range(H):
            kk, vv = k[:, h // (H // KV)], v[:, h // (H // KV)]
            z = np.where(seen, q[:, h] @ kk.T * scale, -np.inf)
            mag = np.where(seen, np.abs(q[:, h]) @ np.abs(kk).T * abs(scale), 0.0)
            p = np.exp(z - z.max(1, keepdims=True))
            p = np.where(seen, p / p.sum(1, keepdims=True), 0.0)
            clean = np.where(np.isfinite(vv), vv, 0.0)
            o, a = p @ clean, p @ np.abs(clean)                       # 0 times NaN is none where a row does not see it
            o[(seen.astype(float) @ (~np.isfinite(vv)).astype(float)) > 0] = np.nan
            # of the weighted sum, and of the sum that it is divided by
            e = 2 * (hd + 4) * 2 * U32 * mag.max(1) + (8 + np.abs(np.where(seen, z, 0.0)).max(1)) * 2 * U32
            e = e[:, None] + (count / 2 + 128) * 2 * U32
            top = np.abs(clean).max(0)
            err[:, :, h] = 2 * e * a + 4 * count * 2.0 ** -126 * top
            err[0, :, h] += 2.0 ** -23 * a
            err[1, :, h] += 2.0 ** -12 * a + count * 2.0 ** -25 * top
            out[:, h] = np.where(some[:, None], o, 0.0)
    err[:, ~some] = 0.0
    return out, err
