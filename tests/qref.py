"""The 8-bit format and the feed-forward operators in float64 NumPy, from the
definitions in include/sd.h: a code is found by comparing against the table of
all e4m3 numbers, a scale by trying powers of two."""
import numpy as np

POS = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])[:127]


def code(v):
    """Bytes of the nearest e4m3 numbers of v (|v| <= 448; ties to the even code; NaN and infinities 0x7f)."""
    v = np.asarray(v, dtype=np.float64)
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    assert a.size == 0 or a.max() <= 448
    hi = np.clip(np.searchsorted(POS, a), 1, 126)
    lo = hi - 1
    up = (POS[hi] - a < a - POS[lo]) | ((POS[hi] - a == a - POS[lo]) & (hi % 2 == 0))
    c = np.where(up, hi, lo) + np.where(np.signbit(v), 128, 0)
    return np.where(np.isfinite(v), c, 0x7f).astype(np.uint8)


def value(c):
    """e4m3 bytes -> float64."""
    c = np.asarray(c, dtype=np.uint8)
    t = np.append(POS, np.nan)[c & 127]
    return np.where(c >= 128, -t, t)


def exponent(amax):
    """Smallest E >= 1 with amax <= 448 2^(E - 127)."""
    amax = np.asarray(amax, dtype=np.float64)
    E = np.ones(amax.shape, dtype=np.int64)
    for k in range(2, 256):
        E = np.where(amax > 448.0 * 2.0 ** (k - 1 - 127), k, E)
    return E


def up(n, m):
    return -(-n // m) * m


def _finite_max(v, axis):
    return np.where(np.isfinite(v), np.abs(v), 0.0).max(axis)


def quantise_rows(y):
    """[M, K] -> (codes [M, K8], E [M, K8 / 128])."""
    M, K = y.shape
    v = np.zeros((M, up(K, 128)))
    v[:, :K] = y
    v = v.reshape(M, -1, 128)
    E = exponent(_finite_max(v, 2))
    return code(v * 2.0 ** (127.0 - E[..., None])).reshape(M, -1), E


def quantise_weight(w):
    """[N, K] -> (codes [N, K], E [N / 128, K / 128])."""
    N, K = w.shape
    v = np.zeros((up(N, 128), up(K, 128)))
    v[:N, :K] = w
    v = v.reshape(v.shape[0] // 128, 128, -1, 128)
    E = exponent(_finite_max(v, (1, 3)))
    return code(v * 2.0 ** (127.0 - E[:, None, :, None])).reshape(up(N, 128), -1)[:N, :K], E


def row_values(codes, E, K):
    M = codes.shape[0]
    return (value(codes).reshape(M, -1, 128) * 2.0 ** (E[..., None] - 127.0)).reshape(M, -1)[:, :K]


def weight_values(codes, E):
    N, K = codes.shape
    s = 2.0 ** (E - 127.0)
    return value(codes) * np.repeat(np.repeat(s, 128, 0)[:N], 128, 1)[:, :K]


def exps_bytes(E):
    out = np.zeros((E.shape[0], up(E.shape[1], 4)), dtype=np.uint8)
    out[:, :E.shape[1]] = E
    return out


def pack(codes, E):
    """The packed bytes, one 16-byte unit at a time."""
    N, K = codes.shape
    c = np.zeros((up(N, 16), up(K, 128)), dtype=np.uint8)
    c[:N, :K] = codes
    out = np.empty((c.shape[0] // 16, c.shape[1] // 128, 128, 16), dtype=np.uint8)
    for h in range(2):
        for g in range(4):
            for r in range(16):
                out[:, :, 64 * h + 16 * g + r] = c[r::16].reshape(c.shape[0] // 16, -1, 128)[:, :, 64 * h + 16 * g:][:, :, :16]
    return np.concatenate([out.reshape(-1), exps_bytes(E).reshape(-1)])


def norm(s, gain, eps):
    return s / np.sqrt(np.mean(s * s, axis=-1, keepdims=True) + eps) * gain


def swiglu(product):
    """[M, 2 F] with gate and up in blocks of 16 -> silu(gate) * up [M, F]."""
    p = product.reshape(product.shape[0], -1, 2, 16)
    g, u = p[:, :, 0].reshape(product.shape[0], -1), p[:, :, 1].reshape(product.shape[0], -1)
    return g / (1.0 + np.exp(-g)) * u
