"""Bounds on the sums of the 8-bit products that do not grow with the number of terms, for terms of random sign.

A sum of K terms t_k is rounded wherever two partial sums are added: inside a block of 128 entries, where partial sums are
about the root of the squares' sum of the block's terms at most, then between blocks, waves and K ranges, where they are about
the root s of all of them.  Each rounding is off by at most a step of fp32, 2^-23 of the partial sum (the matrix unit may
cut), in either direction, so that n of them are off by about the root of n: (root of 128 + root of (K / 128 + 16)) 2^-23 s.
"""
import numpy as np

STEP32 = 2.0 ** -23


def terms(a, w):
    """For values a [M, K], w [N, K]: the products and the roots of their terms' squares' sums, [M, N] both."""
    import torch
    ta, tw = torch.from_numpy(np.ascontiguousarray(a)), torch.from_numpy(np.ascontiguousarray(w))
    return (ta @ tw.T.contiguous()).numpy(), ((ta * ta) @ (tw * tw).T.contiguous()).sqrt().numpy()


def sum_error(K, s):
    return (np.sqrt(128) + np.sqrt(K / 128 + 16)) * STEP32 * s


def cut_error(s):
    """What sums on the 8-bit matrix instruction are off by: measured at 1.4e-5 to 5.1e-5 of s in the 2-norm, over K of 128 to
    11008 and rows with and without large entries; this is 2.4 times the largest."""
    return 2.0 ** -13 * s


def to_bf16(v):
    """float64 -> the nearest bf16 (ties to even), as float64; for magnitudes that are normal numbers or zero."""
    m, e = np.frexp(v)
    return np.ldexp(np.round(m * 256), e - 8)


def _tiles(a, size=128):
    for i in range(0, a.shape[0], size):
        for j in range(0, a.shape[1], size):
            yield slice(i, i + size), slice(j, j + size)


def product_ok(got, want, err, dtype):
    """err: what the sums may be off by (the bound's size for one of them).  fp32: in every tile of the output the 2-norm of
    the difference is within err's.  bf16: every output is the rounding of a number within 16 err of the sum; and outputs that
    round the other way, by a step of at most 2^-7 |v|, are those whose border lies inside the error, a share e / step
    of them, which makes a squared difference of e 2^-7 |v|."""
    d = np.abs(got - want)
    if not np.isfinite(d).all():
        return False
    if dtype == "fp32":
        return all(np.linalg.norm(d[t]) <= np.linalg.norm(err[t]) for t in _tiles(d))
    if ((got < to_bf16(want - 16 * err)) | (got > to_bf16(want + 16 * err))).any():
        return False
    return np.linalg.norm(got - to_bf16(want)) <= np.sqrt(2.0 ** -7 * np.linalg.norm(err) * np.linalg.norm(want))


def swiglu_error(product, err):
    """What silu(gate) up is off by where gate and up are off by err: |silu'| <= 1.1, and eight steps for its own arithmetic."""
    p, e = (x.reshape(x.shape[0], -1, 2, 16) for x in (product, err))
    g, u, dg, du = (x.reshape(x.shape[0], -1) for x in (p[:, :, 0], p[:, :, 1], e[:, :, 0], e[:, :, 1]))
    silu = np.abs(g / (1 + np.exp(-g)))
    return np.sqrt((1.1 * dg * u) ** 2 + (silu * du) ** 2) + 8 * STEP32 * silu * np.abs(u)


def codes_ok(values, h, err, want, scale):
    """Codes' values of h, known to about err: every one is within half a step (2^-4 of it, or 2^-10 scales among the
    smallest codes) of a number within 16 err of h; and those that are another code than h's are the share whose border lies
    inside the error, steps of at most 2^-3 |h| + 2^-9 scales.  want: the values of h's own codes."""
    if not np.isfinite(values).all():
        return False
    far = 16 * err + np.maximum(2.0 ** -4 * (np.abs(h) + 16 * err), 2.0 ** -10 * scale)
    if (np.abs(values - h) > far).any():
        return False
    return np.linalg.norm(values - want) <= np.sqrt(np.linalg.norm(err) * np.linalg.norm(2.0 ** -3 * np.abs(h) + 2.0 ** -9 * scale))
