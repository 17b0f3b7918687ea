"""Attention over the 4-bit cache at the ends of its numbers' range: scores, weights and values."""
import numpy as np
import pytest

import kvplans
from kvref import HALF
from sdcase import say
from test_gpu_kv_q import Case, close, host, t

pytestmark = pytest.mark.gpu

KERNELS = [  # name, rows, lengths, heads, kv heads, head_dim, type, pages that the table is wide, plan
    ("one key", [1], [1], 4, 2, 64, "bf16", 1, (0, 16, 8, 1, 0)),
    ("one key, fp32", [1], [1], 4, 2, 128, "fp32", 1, (0, 16, 8, 1, 0)),
    ("waves of 8", [5, 1, 3], [600, 33, 1000], 8, 2, 128, "bf16", 64, (0, 16, 8, 1, 0)),
    ("waves of 8, fp32", [5, 1, 3], [600, 33, 1000], 8, 2, 64, "fp32", 64, (0, 16, 8, 1, 0)),
    ("two tiles", [9] * 16, [9 + 37 * i for i in range(16)], 32, 8, 128, "bf16", 150, (0, 32, 4, 1, 0)),
    ("key ranges", [2], [9000], 16, 2, 64, "bf16", 600, (0, 16, 4, 37, 0)),
    ("key ranges, fp32", [3], [1500], 16, 4, 64, "fp32", 110, (0, 16, 4, 6, 0)),
    ("shared", [520, 520], [700, 555], 32, 16, 128, "bf16", 44, (1, 128, 4, 1, 0)),
    ("shared, 64 dimensions", [520, 520], [700, 555], 32, 16, 64, "bf16", 44, (1, 128, 4, 1, 0)),
]
kernels = pytest.mark.parametrize("kernel", KERNELS, ids=lambda k: k[0])


def case_of(r, kernel):
    name, rows, lengths, H, KV, hd, dtype, width, plan = kernel
    assert kvplans.plan(sum(rows), H, KV, hd, dtype, len(rows), 16 * width) == plan
    return Case(r, rows, lengths, KV, hd, width=width), H, dtype


def put(c, b, k, v):
    c.pool.put(*c.at(b, np.arange(c.lengths[b])), k.astype(np.float32), v.astype(np.float32))


@kernels
@pytest.mark.parametrize("power", [17, 21, 24, 25, 26, 29, 33, 40, 100])
@pytest.mark.parametrize("scale", [1.0, -0.37])
def test_large_scores(kernel, power, scale):
    """Scores from 2^17 on that are exact in fp32 and lie far apart or are equal: the output is the mean of the values whose
    scores are the largest.

    Equal scores have equal weights.  bf16 calls enter a weight into the product as two bf16 parts, off by 2^-15 of it;
    fp32 ones as it is.  The kernel that shares its keys enters it as one fp16 number, off by 2^-11 of it, but for a
    workgroup's last keys: weights (1 + d) w with |d| <= 2^-11 make a mean that is off by at most 2 2^-11 / (1 - 2^-11) of the
    mean of the values' magnitudes, a little over 2^-10.  The sums of n weights and of n values are of as many roundings,
    their quotient of two more."""
    from paper_2510_11331_amd import attention_q
    say("large scores", kernel[0], power, scale)
    r = np.random.default_rng([power, len(kernel[0])])
    c, H, dtype = case_of(r, kernel)
    KV, hd, G = c.KV, c.hd, H // c.KV
    numbers = np.array([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6])
    q = np.zeros((c.M, H, hd))
    q[:, :, 5] = r.choice([-1.75, -1.5, -1.0, 1.0, 1.25, 1.5], size=(c.M, H)) * 2.0 ** power
    want, far = np.zeros(q.shape), np.zeros(q.shape)
    for b, (n, m) in enumerate(zip(c.rows, c.lengths)):
        k, v = np.zeros((m, KV, hd)), r.choice(numbers, size=(m, KV, hd))
        k[:, :, 5] = r.choice(numbers, size=(m, KV))
        put(c, b, k, v)
        s = slice(c.cu[b], c.cu[b] + n)
        seen = np.arange(m)[None] <= c.pos[s][:, None]
        for h in range(H):
            z = np.where(seen, np.sign(scale) * q[s, h, 5][:, None] * k[:, h // G, 5][None], -np.inf)
            top = (z == z.max(1, keepdims=True)).astype(float)
            count = top.sum(1, keepdims=True)
            want[s, h] = top @ v[:, h // G] / count
            a = top @ np.abs(v[:, h // G]) / count
            form = 0.0 if dtype == "fp32" else 2.0 ** -14 if kernel[8][0] == 0 else 1.001 * 2.0 ** -10
            far[s, h] = a * form + a * (count + 4) * 2.0 ** -23
    got = host(attention_q(t(q.astype(np.float32), dtype), c.cache(), c.desc, scale=scale))
    bad = ~(np.abs(got - want) <= far + np.abs(want) * HALF[dtype] * 1.001)
    assert not bad.any(), (bad.sum(), np.isnan(got).sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


@kernels
@pytest.mark.parametrize("power", [10, 16, 18, 20, 21, 22])
@pytest.mark.parametrize("scale", [1.0, -0.7])
def test_close_scores(kernel, power, scale):
    """Scores that lie by 0 to 12 apart at 2^power, all of them exact in fp32: the weights are those of the differences.

    What the logarithm of a weight is off by does not depend on the scores' size: a rounding of itself, and the two of its
    factor scale log2(e), 2^-22 of 12 1.5 or less; the exponential and a move of the maximum are off by a few steps more, so
    that 2^-17 holds them all twice over.  The forms of a weight are those of the test above."""
    from paper_2510_11331_amd import attention_q
    say("close scores", kernel[0], power, scale)
    r = np.random.default_rng([power, len(kernel[0])])
    c, H, dtype = case_of(r, kernel)
    KV, hd, G = c.KV, c.hd, H // c.KV
    numbers = np.array([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6])
    q = np.zeros((c.M, H, hd))
    q[:, :, 5], q[:, :, 40] = r.choice([-1, 1], size=(c.M, H)) * 2.0 ** power, r.choice([-1, 1], size=(c.M, H))
    want, far = np.zeros(q.shape), np.zeros(q.shape)
    for b, (n, m) in enumerate(zip(c.rows, c.lengths)):
        k, v = np.zeros((m, KV, hd)), r.choice(numbers, size=(m, KV, hd))
        k[:, :, 5], k[:, :, 40] = 1, r.choice(numbers, size=(m, KV))
        put(c, b, k, v)
        s = slice(c.cu[b], c.cu[b] + n)
        seen = np.arange(m)[None] <= c.pos[s][:, None]
        for h in range(H):
            d = q[s, h, 40][:, None] * k[:, h // G, 40][None] * scale
            w = np.where(seen, np.exp(d - np.where(seen, d, -np.inf).max(1, keepdims=True)), 0.0)
            w /= w.sum(1, keepdims=True)
            want[s, h] = w @ v[:, h // G]
            form = 0.0 if dtype == "fp32" else 2.0 ** -14 if kernel[8][0] == 0 else 1.001 * 2.0 ** -10
            far[s, h] = (w @ np.abs(v[:, h // G])) * (form + 2.0 ** -16 + (seen.sum(1, keepdims=True) / 2 + 128) * 2.0 ** -22)
    got = host(attention_q(t(q.astype(np.float32), dtype), c.cache(), c.desc, scale=scale))
    bad = ~(np.abs(got - want) <= far + np.abs(want) * HALF[dtype] * 1.001)
    assert not bad.any(), (bad.sum(), np.isnan(got).sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


@kernels
@pytest.mark.parametrize("size", [1e5, 1e7, 1e9, 1e10, 1e14, 1e30])
def test_large_scores_of_any_query(kernel, size):
    """Any finite scores: every dimension of an output lies between the smallest and the largest of the values seen, but
    for the roundings of weights (2^-11 at most, 2^-10 of the values with their sum's), sums and outputs."""
    from paper_2510_11331_amd import attention_q
    say("any large scores", kernel[0], size)
    r = np.random.default_rng([int(np.log2(size)), len(kernel[0])])
    c, H, dtype = case_of(r, kernel)
    G = H // c.KV
    q = t((r.normal(size=(c.M, H, c.hd)) * np.exp(r.normal(size=(c.M, H, 1)))).astype(np.float32), dtype)
    lo, hi = np.zeros(q.shape), np.zeros(q.shape)
    for b, (n, m) in enumerate(zip(c.rows, c.lengths)):
        x = r.normal(size=(2, m, c.KV, c.hd))
        put(c, b, x[0], x[1])
        v = c.pool.get(*c.at(b, np.arange(m)))[1]
        s, pos = slice(c.cu[b], c.cu[b] + n), c.pos[c.cu[b]:c.cu[b] + n]
        lo[s], hi[s] = (np.repeat(f.accumulate(v)[pos], G, 1) for f in (np.minimum, np.maximum))
    for scale in (size, -size):
        got = host(attention_q(q, c.cache(), c.desc, scale=scale))
        slack = np.maximum(np.abs(lo), np.abs(hi)) * (2.0 ** -10 + HALF[dtype])
        bad = ~((got >= lo - slack) & (got <= hi + slack))
        assert not bad.any(), (bad.sum(), np.isnan(got).sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], lo[bad][:4], hi[bad][:4])


@kernels
def test_large_values(kernel):
    """Values of up to 2^96: outputs between the smallest and the largest of those seen, as above."""
    from paper_2510_11331_amd import attention_q
    say("large values", kernel[0])
    r = np.random.default_rng(len(kernel[0]))
    c, H, dtype = case_of(r, kernel)
    q = t(r.normal(size=(c.M, H, c.hd)).astype(np.float32), dtype)
    lo, hi = np.zeros(q.shape), np.zeros(q.shape)
    for b, (n, m) in enumerate(zip(c.rows, c.lengths)):
        x = r.normal(size=(2, m, c.KV, c.hd))
        put(c, b, 4 * x[0], np.clip(x[1] / 2, -1, 1) * 2.0 ** 95.9)
        v = c.pool.get(*c.at(b, np.arange(m)))[1]
        s, pos = slice(c.cu[b], c.cu[b] + n), c.pos[c.cu[b]:c.cu[b] + n]
        lo[s], hi[s] = (np.repeat(f.accumulate(v)[pos], H // c.KV, 1) for f in (np.minimum, np.maximum))
    got = host(attention_q(q, c.cache(), c.desc))
    slack = np.maximum(np.abs(lo), np.abs(hi)) * (2.0 ** -10 + HALF[dtype])
    bad = ~((got >= lo - slack) & (got <= hi + slack))
    assert not bad.any(), (bad.sum(), np.isnan(got).sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], lo[bad][:4], hi[bad][:4])


@kernels
@pytest.mark.parametrize("E", [252, 253, 254])
def test_values_at_the_end_of_the_range(kernel, E):
    """Tokens of the pass's own rows with 6 2^(E - 127) and its negative among 32 zeros: from E = 253 on these are infinities
    in bf16 and fp32.  They reach no output but the rows' that see the token, in their dimension."""
    from paper_2510_11331_amd import attention_q
    say("end of the range", kernel[0], E)
    r = np.random.default_rng([E, len(kernel[0])])
    c, H, dtype = case_of(r, kernel)
    c.fill(r)
    KV, hd, G = c.KV, c.hd, H // c.KV
    q = t(r.normal(size=(c.M, H, hd)).astype(np.float32), dtype)
    put_in, reached = [], np.zeros((c.M, H, hd), bool)
    for b, (n, m) in enumerate(zip(c.rows, c.lengths)):
        for pos in np.unique(m - n + r.integers(min(1, n - 1), n, size=3)):
            page, tok = c.at(b, pos)
            kvh, block, dims = r.integers(KV), r.integers(hd // 32), r.choice(16, size=2, replace=False) * 2
            bytes_of = c.pool.bytes[page, kvh]
            codes = c.pool.vc[tok, block * 16:block * 16 + 16]
            bytes_of[codes] = 0
            bytes_of[c.pool.vs[tok, block]] = 127
            put_in.append((bytes_of, codes[dims // 2], c.pool.vs[tok, block]))
            rows = c.cu[b] + np.arange(n)[c.pos[c.cu[b]:c.cu[b] + n] >= pos]
            reached[np.ix_(rows, np.arange(kvh * G, kvh * G + G), block * 32 + dims)] = True
    want, err = c.attention(host(q))
    for bytes_of, codes, scale in put_in:
        bytes_of[codes] = 7, 15
        bytes_of[scale] = E
    got = host(attention_q(q, c.cache(), c.desc))
    close(got[~reached], want[~reached], err[:, ~reached], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_appended_values_at_the_end_of_the_range(hd, dtype):
    """What would be rounded to an infinity is kept as an infinity is, as NaN, and reaches the rows that see it only; the
    next smaller value is a number."""
    from paper_2510_11331_amd import attention_q, kv_append_q, kv_read_q
    say("appended at the range's end", hd, dtype)
    r = np.random.default_rng(hd)
    end = 1.75 * 2.0 ** 127
    below = end * (1 - 2.0 ** -8) if dtype == "bf16" else float(np.nextafter(np.float32(end), np.float32(0)))
    for value, is_nan in ((1.9 * 2.0 ** 127, True), (-end, True), (-below, False)):
        c = Case(r, [20], [50], 2, hd)
        c.fill(r)
        x = t(r.normal(size=(2, 20, 2, hd)).astype(np.float32), dtype)
        x[1, 19, 1, 40] = value
        x[0, 18, 0, hd - 1] = value
        cache = c.cache()
        kv_append_q(cache, x[0], x[1], c.desc)
        got = [host(y) for y in kv_read_q(cache, c.desc, 20, x.dtype)]
        v = got[1][19, 1, 32:64]
        k = got[0][18, 0, hd - 32:]
        if is_nan:
            assert np.isnan(v).all() and np.isnan(k).all()
        else:
            assert v[8] == k[31] == -1.5 * 2.0 ** 127 and (np.delete(v, 8) == 0).all() and (k[:31] == 0).all()
        assert np.isfinite(got[1][:19]).all() and np.isfinite(got[0][:18]).all() and np.isfinite(got[0][19]).all()
        q = t(r.normal(size=(20, 4, hd)).astype(np.float32), dtype)
        page, tok = c.at(0, np.array([48, 49]))
        c.pool.bytes[:] = cache.data.cpu().numpy()
        c.pool.bytes[page[0], 0, c.pool.ks[tok[0], -1]] = c.pool.bytes[page[1], 1, c.pool.vs[tok[1], 1]] = 1   # for the reference
        want, err = c.attention(host(q))
        out = host(attention_q(q, cache, c.desc))
        ok = np.ones(out.shape, bool)
        ok[18:, :2] = False                                              # that key's rows
        ok[19, 2:, 32:64] = False                                        # that value's
        close(out[ok], want[ok], err[:, ok], dtype)
        if is_nan:
            assert np.isnan(out[18:, :2]).all() and np.isnan(out[19, 2:, 32:64]).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("kernel", ["shared", "waves of 8"])
@pytest.mark.parametrize("power", [13, 22.6, 24.4, 26.7])
def test_many_small_weights(kernel, hd, power):
    """One key outweighs each of the others by 2^power, and its value is zero: the outputs are what the others' weights add up
    to.

    A weight of the kernel that shares its keys is one fp16 number, 2^7 of the largest: off by 2^-11 of it, or by 2^-32 of
    the largest where it is below fp16's normal numbers (half of 2^-24, of 2^7); relative errors of the weights are the
    outputs' twice over, with the sum that they are divided by.  Elsewhere it is two bf16 parts, off by 2^-15.  The scores are
    of one product; with their scale and the exponential's argument they are off by a few roundings of 27, 2^-18 in all."""
    from paper_2510_11331_amd import attention_q
    say("small weights", kernel, hd, power)
    r = np.random.default_rng([hd, int(10 * power)])
    rows, lengths, H, KV, shared = ([520, 520], [3900, 2970], 32, 16, 1) if kernel == "shared" else ([2, 2], [3900, 2970], 32, 16, 0)
    c = Case(r, rows, lengths, KV, hd)
    assert kvplans.plan(sum(rows), H, KV, hd, "bf16", 2, 16 * c.table.shape[1])[0] == shared
    for b, m in enumerate(lengths):
        k, v = np.zeros((m, KV, hd)), r.choice([0.5, 1, 1.5, 2, 3, 4, 6], size=(m, KV, hd)) * r.choice([1, -1], size=(1, KV, hd))
        k[0, :, 5], v[0] = 6, 0
        put(c, b, k, v)
    q = np.zeros((c.M, H, hd))
    q[:, :, 5] = 1
    got = host(attention_q(t(q.astype(np.float32), "bf16"), c.cache(), c.desc, scale=power * np.log(2) / 6))
    for b, (n, m) in enumerate(zip(rows, lengths)):
        v = c.pool.get(*c.at(b, np.arange(m)))[1]
        sums, count = np.cumsum(v, 0), np.arange(m)[:, None, None]
        want = (sums / (2.0 ** power + count))[m - n:].repeat(H // KV, 1)
        here = got[c.cu[b]:c.cu[b] + n]
        slack = np.abs(want) * (2 * (2.0 ** -11 if shared else 2.0 ** -15) + 2.0 ** -18 + (m / 2 + 128) * 2.0 ** -23 + HALF["bf16"])
        slack += shared * 2.0 ** -32 * m * 6
        bad = ~(np.abs(here - want) <= slack * 1.001)
        assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), here[bad][:4], want[bad][:4], slack[bad][:4])
