"""The 4-bit cache's operators against their definitions in float64 (kvref)."""
import numpy as np
import pytest

import kvplans
import kvref
from kvref import HALF, U32
from sdcase import say

pytestmark = pytest.mark.gpu


def t(a, dtype=None):
    import torch
    x = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return x if dtype is None else x.to(dt(dtype))


def dt(name):
    import torch
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


def host(x):
    return x.double().cpu().numpy()


def heads(r, M, H, hd, dtype):
    """Values of a type as a tensor and in float64."""
    x = t((r.normal(size=(M, H, hd)) * np.exp(0.5 * r.normal(size=(M, H, 1)))).astype(np.float32), dtype)
    return x, host(x)


class Case:
    """Sequences with pages in random order, one more page between them, table entries behind the last page bad."""

    def __init__(self, r, rows, lengths, KV, hd, extra=3, fill=0xff, width=None):
        from paper_2510_11331_amd import KVRows
        self.rows, self.lengths, self.KV, self.hd = rows, lengths, KV, hd
        used = [-(-max(n, 0) // 16) for n in lengths]
        blocks = sum(used) + extra
        order = r.permutation(blocks)
        W = width or max(1, max(used))
        self.table = np.array([-1, blocks, 1 << 30, -(1 << 30)], dtype=np.int32)[r.integers(0, 4, size=(len(rows), W))]
        at = 0
        for b, n in enumerate(used):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.M = int(self.cu[-1])
        self.b, self.pos = kvref.places(rows, lengths)
        self.pool = kvref.Pool(blocks, KV, hd, fill)
        self.desc = KVRows(t(self.cu), t(np.array(lengths, dtype=np.int32)), t(self.table))

    def at(self, b, pos):
        return self.table[b, pos // 16], pos % 16

    def fill(self, r, sizes=1.0):
        """All positions get keys and values."""
        for b, n in enumerate(self.lengths):
            if n <= 0:
                continue
            p = np.arange(n)
            x = r.normal(size=(2, len(p), self.KV, self.hd)).astype(np.float32) * sizes
            self.pool.put(*self.at(b, p), x[0], x[1])

    def cache(self):
        from paper_2510_11331_amd import KVCacheQ
        return KVCacheQ(t(self.pool.bytes))

    def attention(self, q, causal=True, scale=None):
        """(out, err) of all rows."""
        out, err = np.zeros(q.shape), np.zeros((2, *q.shape))
        scale = self.hd ** -0.5 if scale is None else scale
        for b, (n, m) in enumerate(zip(self.rows, self.lengths)):
            if not n:
                continue
            m = max(m, 0)
            k, v = self.pool.get(*self.at(b, np.arange(m)))
            s = slice(self.cu[b], self.cu[b] + n)
            seen = np.arange(m)[None] <= (self.pos[s] if causal else np.full(n, m))[:, None]
            out[s], err[:, s] = kvref.attention(q[s], k, v, seen, scale)
        return out, err


def close(got, want, err, dtype):
    """Within the arithmetic's error and the output's rounding."""
    far = err[("fp32", "bf16").index(dtype)] + np.abs(want) * HALF[dtype] * 1.001
    bad = ~((np.abs(got - want) <= far) | (np.isnan(got) & np.isnan(want)) | (got == want))
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], far[bad][:4])


# ------------------------------------------------------------------ writing and reading

SEQS = [([1], [1]), ([5, 0, 3], [37, 9, 3]), ([17, 1, 16, 33], [17, 2049, 64, 50]), ([2] * 70, [40 + i for i in range(70)])]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,KV", [(64, 1), (128, 3), (64, 8), (128, 8)])
@pytest.mark.parametrize("rows,lengths", SEQS)
def test_append_and_read(rows, lengths, hd, KV, dtype):
    """The pool byte for byte, what no row writes included; and read back, exactly."""
    from paper_2510_11331_amd import kv_append_q, kv_read_q
    say("append", rows, lengths, hd, KV, dtype)
    r = np.random.default_rng([hd, KV, len(rows)])
    c = Case(r, rows, lengths, KV, hd)
    (k, k64), (v, v64) = heads(r, c.M, KV, hd, dtype), heads(r, c.M, KV, hd, dtype)
    cache = c.cache()
    kv_append_q(cache, k, v, c.desc)
    c.pool.put(*c.at(c.b, c.pos), k64, v64)
    assert np.array_equal(cache.data.cpu().numpy(), c.pool.bytes)
    want = c.pool.get(*c.at(c.b, c.pos))
    got = kv_read_q(cache, c.desc, c.M, dt(dtype))
    assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])


@pytest.mark.parametrize("hd", [64, 128])
def test_append_special_values(hd):
    """Blocks of zeros of both signs, of fp32's smallest and largest numbers, at the scale's border, of ties and next to
    them, with NaN and infinities."""
    from paper_2510_11331_amd import kv_append_q, kv_read_q
    say("append special", hd)
    r = np.random.default_rng(hd)
    n = 24
    c = Case(r, [n], [n], 1, hd)
    x = r.normal(size=(n, 1, hd)).astype(np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 6.0, -0.25, -5.0], dtype=np.float32)
    x[0] = 0
    x[1] = -0.0
    x[2] *= 1e-38
    x[3] *= 2.0 ** -149 * 3
    x[4] = 2.0 ** -149
    x[5, 0, 3] = 2.0 ** 127 * 1.74
    x[6, 0, 3] = np.nan
    x[7, 0, hd - 1] = np.inf
    x[8, 0, 40] = -np.inf
    for i, e in enumerate((-126, -100, -3, 0, 1, 60, 122)):
        x[9 + i, 0] = np.resize(ties, hd) * np.float32(2.0 ** e)
        x[9 + i, 0, ::32] = 6 * np.float32(2.0 ** e)                      # the scale's border stays
    x[16, 0] = np.nextafter(np.resize(ties, hd), np.float32(9))
    x[17, 0] = np.nextafter(np.resize(ties, hd), np.float32(-9))
    x[18, 0] = 6
    x[19, 0] = np.nextafter(np.float32(6), np.float32(9))
    x[20, 0] = 6 * 2.0 ** -126
    x[21, 0] = np.nextafter(np.float32(6 * 2.0 ** -126), np.float32(1))
    cache = c.cache()
    v = x[::-1].copy()
    kv_append_q(cache, t(x), t(v), c.desc)
    c.pool.put(*c.at(c.b, c.pos), x, v)
    assert np.array_equal(cache.data.cpu().numpy(), c.pool.bytes)
    for got, want in zip(kv_read_q(cache, c.desc, n, dt("fp32")), c.pool.get(*c.at(c.b, c.pos))):
        assert np.array_equal(host(got), want, equal_nan=True)


def test_rows_without_places():
    """Rows before the first position, behind the table, on bad pages, behind the last sequence: not written, read as
    NaN, the last ones left as they were."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q
    say("rows without places")
    hd, KV = 64, 2
    r = np.random.default_rng(1)
    table = np.array([[3, -1, 1], [0, 4, 6], [2, 5, 7]], dtype=np.int32)     # of 6 pages
    rows, lengths = [8, 40, 20], [3, 40, 50]                                 # -5 .. 2; 0 .. 39; 30 .. 49
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    M = 75                                                                   # seven more rows
    desc = KVRows(t(cu), t(np.array(lengths, dtype=np.int32)), t(table))
    pool = kvref.Pool(6, KV, hd)
    cache = KVCacheQ(t(pool.bytes))
    (k, k64), (v, v64) = heads(r, M, KV, hd, "fp32"), heads(r, M, KV, hd, "fp32")
    b, pos = kvref.places(rows, lengths)
    has = (pos >= 0) & (pos < 48)
    page = np.where(has, table[b, np.clip(pos, 0, 47) // 16], -1)
    has &= (page >= 0) & (page < 6)
    pool.put(page[has], pos[has] % 16, k64[:68][has], v64[:68][has])
    kv_append_q(cache, k, v, desc)
    assert np.array_equal(cache.data.cpu().numpy(), pool.bytes)
    for got, want in zip(kv_read_q(cache, desc, M, torch.float32, torch.full((M, KV, hd), 7.0, device="cuda"),
                                   torch.full((M, KV, hd), 7.0, device="cuda")), pool.get(page.clip(0, 5), pos % 16)):
        want[~has] = np.nan
        assert np.array_equal(host(got)[:68], want, equal_nan=True) and (host(got)[68:] == 7).all()
    # a row that sees a position without a page is NaN; rows that see none of these are not
    q, q64 = heads(r, M, 4, hd, "fp32")
    out = attention_q(q, cache, desc, out=torch.full((M, 4, hd), 7.0, device="cuda"))
    got = host(out)
    assert (got[68:] == 7).all()
    assert (got[:5] == 0).all() and np.isfinite(got[5:8]).all()              # nothing to see; the first 3 positions
    assert np.isfinite(got[8:40]).all() and np.isnan(got[40:48]).all()       # page 6 is none
    assert np.isnan(got[48:68]).all()                                        # page 5 was not written in whole, 7 is none


def test_strided_rows():
    """Views of one QKV product, and outputs with strides; what lies between is not written."""
    import torch
    from paper_2510_11331_amd import attention_q, kv_append_q, kv_read_q, norm_rope, norm_rope_append_q, rope_table
    say("strides")
    r = np.random.default_rng(2)
    H, KV, hd = 6, 2, 128
    c = Case(r, [5, 7], [50, 7], KV, hd)
    c.fill(r)
    qkv = t(r.normal(size=(c.M, (H + 2 * KV) * hd + 8)).astype(np.float32), "bf16")
    at = lambda a, n: qkv[:, a * hd:(a + n) * hd].unflatten(1, (n, hd))
    q, k, v = at(0, H), at(H, KV), at(H + KV, KV)
    rope, gain = rope_table(64, hd), t((1 + 0.1 * r.normal(size=hd)).astype(np.float32))
    a, b = c.cache(), c.cache()
    kv_append_q(a, k, v, c.desc)
    kv_append_q(b, k.contiguous(), v.contiguous(), c.desc)
    assert torch.equal(a.data, b.data)
    wide = lambda n: torch.full((c.M, n * hd + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    wq, wk, wv, wo = wide(H), wide(KV), wide(KV), wide(H)
    view = lambda w, n: w[:, 8:8 + n * hd].unflatten(1, (n, hd))
    pos = t(c.pos.astype(np.int32))
    x = norm_rope(q, k, pos, rope, gain, gain, q_out=view(wq, H), k_out=view(wk, KV))
    y = norm_rope(q.contiguous(), k.contiguous(), pos, rope, gain, gain)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1]) and x[0].data_ptr() == wq[:, 8:].data_ptr()
    assert torch.equal(norm_rope_append_q(a, q, k, v, c.desc, rope, gain, gain, q_out=view(wq, H)), y[0])
    norm_rope_append_q(b, q.contiguous(), k.contiguous(), v.contiguous(), c.desc, rope, gain, gain)
    assert torch.equal(a.data, b.data)
    x = kv_read_q(a, c.desc, c.M, k_out=view(wk, KV), v_out=view(wv, KV))
    y = kv_read_q(a, c.desc, c.M)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    assert torch.equal(attention_q(q, a, c.desc, out=view(wo, H)), attention_q(q.contiguous(), a, c.desc))
    for w, n in ((wq, H), (wk, KV), (wv, KV), (wo, H)):
        assert (w[:, :8] == 7).all() and (w[:, 8 + n * hd:] == 7).all()
    # in place
    want = norm_rope(q, k, pos, rope, gain, gain)
    x = norm_rope(q, k, pos, rope, gain, gain, q_out=q, k_out=k)
    assert x[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])


# ------------------------------------------------------------------ norms and rotation


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,H,KV,hd", [(1, 1, 1, 64), (3, 4, 2, 128), (129, 32, 8, 64), (67, 5, 5, 128)])
@pytest.mark.parametrize("gains", ["bf16", "fp32", None, "q"])
@pytest.mark.parametrize("rotate", [True, False])
def test_norm_rope(M, H, KV, hd, dtype, gains, rotate):
    """Rounded to fp32, and from there to the type: off by at most half a step of each of the two."""
    from paper_2510_11331_amd import norm_rope, rope_table
    say("norm_rope", M, H, KV, hd, dtype, gains, rotate)
    r = np.random.default_rng([M, H, hd])
    (q, q64), (k, k64) = heads(r, M, H, hd, dtype), heads(r, M, KV, hd, dtype)
    gt = "fp32" if gains == "q" else gains
    gq = t((1 + 0.1 * r.normal(size=hd)).astype(np.float32), gt) if gains else None
    gk = t((1 + 0.1 * r.normal(size=hd)).astype(np.float32), gt) if gains and gains != "q" else None
    n_pos = 5000
    rope = rope_table(n_pos, hd, 500.0) if rotate else None
    pos = r.integers(0, n_pos, size=M).astype(np.int32)
    pos[0] = n_pos - 1
    got = norm_rope(q, k, t(pos) if rotate else None, rope, gq, gk, 1e-6)
    cs = host(rope)[pos] if rotate else None
    for g, x, w in ((got[0], q64, gq), (got[1], k64, gk)):
        want = kvref.norm_rope(x, None if w is None else host(w), cs, 1e-6)
        # a rotation's difference may be small against what it is taken of: 64 bits leave 2^-50 of that
        slack = 2.0 ** -50 * (np.abs(x).max() + 10) * 10
        assert (np.abs(host(g) - want) <= np.abs(want) * (HALF[dtype] + (U32 if dtype == "bf16" else 0)) * 1.0001 + slack + 2.0 ** -149).all()


@pytest.mark.parametrize("gains", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_gain_addresses(hd, gains):
    """A gain is aligned to its entries only: the same result from any of them."""
    import torch
    from paper_2510_11331_amd import norm_rope
    say("gain addresses", hd, gains)
    r = np.random.default_rng(hd)
    (q, _), (k, _) = heads(r, 7, 4, hd, "bf16"), heads(r, 7, 2, hd, "bf16")
    g = t((1 + 0.1 * r.normal(size=hd)).astype(np.float32), gains)
    want = norm_rope(q, k, q_gain=g, k_gain=g)
    for at in range(1, 9):
        room = torch.full((hd + 16,), float("nan"), dtype=g.dtype, device="cuda")
        room[at:at + hd] = g
        got = norm_rope(q, k, q_gain=room[at:at + hd], k_gain=room[at:at + hd])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_values_that_are_not_finite():
    """Without a norm and a rotation a head's entries are what they were; a rotation mixes the two of a pair only."""
    import torch
    from paper_2510_11331_amd import norm_rope, rope_table
    say("not finite")
    q = torch.arange(128, dtype=torch.float32, device="cuda").repeat(3, 2, 1).contiguous()
    q[0, 0, 3], q[0, 1, 70], q[1, 0, 127], q[2, 1, 0] = float("inf"), float("-inf"), float("nan"), -0.0
    got = norm_rope(q, q[:, :1].contiguous())
    assert torch.equal(torch.isnan(got[0]), torch.isnan(q))
    assert torch.equal(got[0].nan_to_num(5.0, 6.0, 7.0).view(torch.int32), q.nan_to_num(5.0, 6.0, 7.0).view(torch.int32))
    got = norm_rope(q, q[:, :1].contiguous(), torch.ones(3, dtype=torch.int32, device="cuda"), rope_table(2, 128))[0]
    bad = torch.zeros(3, 2, 128, dtype=torch.bool, device="cuda")
    for row, h, d in ((0, 0, 3), (0, 1, 6), (1, 0, 63)):
        bad[row, h, d] = bad[row, h, d + 64] = True
    assert torch.equal(~torch.isfinite(got), bad)


def test_rope_table():
    from paper_2510_11331_amd import rope_table
    say("rope table")
    for n, hd, theta in ((40000, 128, 10000.0), (7, 64, 1e6)):
        a = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
        got = host(rope_table(n, hd, theta))
        # the angle in 64 bits is off by a few 2^-53 of itself, its functions by that
        assert np.abs(got - np.stack([np.cos(a), np.sin(a)], -1)).max() <= U32 + 4 * 2.0 ** -52 * n


def test_positions_outside_the_table():
    """They make NaN, of their rows only; NaN and infinities in a head stay in it."""
    from paper_2510_11331_amd import norm_rope, rope_table
    say("positions outside")
    r = np.random.default_rng(3)
    (q, q64), (k, k64) = heads(r, 6, 2, 64, "fp32"), heads(r, 6, 1, 64, "fp32")
    q[4, 1, 5], k[5, 0, 63] = float("nan"), float("inf")
    g = t(np.ones(64, dtype=np.float32))
    q, k = norm_rope(q, k, t(np.array([0, -1, 9, 10, 1, 2], dtype=np.int32)), rope_table(10, 64), g, g)
    bad = np.isnan(host(q)).all(-1)
    assert np.array_equal(bad, [[0, 0], [1, 1], [0, 0], [1, 1], [0, 1], [0, 0]]) and np.isfinite(host(q)[~bad]).all()
    assert np.isnan(host(k)[[1, 3]]).all() and np.isfinite(host(k)[[0, 2, 4]]).all() and np.isnan(host(k)[5]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,KV,hd", [(2, 1, 64), (3, 3, 128), (32, 8, 64)])
def test_norm_rope_append(H, KV, hd, dtype):
    """The queries are norm_rope's; the pool is that of the keys' fp32 values, byte for byte."""
    import torch
    from paper_2510_11331_amd import norm_rope, norm_rope_append_q, rope_table
    say("norm_rope_append", H, KV, hd, dtype)
    r = np.random.default_rng([H, hd])
    c = Case(r, [5, 0, 20, 1], [37, 4, 20, 300], KV, hd)
    (q, q64), (k, k64), (v, v64) = (heads(r, c.M, n, hd, dtype) for n in (H, KV, KV))
    gq, gk = (t((1 + 0.1 * r.normal(size=hd)).astype(np.float32), "bf16") for _ in range(2))
    rope = rope_table(300, hd)
    cache = c.cache()
    got = norm_rope_append_q(cache, q, k, v, c.desc, rope, gq, gk, 1e-5)
    assert torch.equal(got, norm_rope(q, k, t(c.pos.astype(np.int32)), rope, gq, gk, 1e-5)[0])
    k64 = kvref.norm_rope(k64, host(gk), host(rope)[c.pos], 1e-5).astype(np.float32)
    c.pool.put(*c.at(c.b, c.pos), k64, v64)
    assert np.array_equal(cache.data.cpu().numpy(), c.pool.bytes)


# ------------------------------------------------------------------ attention

ATTN = [  # rows, lengths, H, KV
    ([1], [1], 1, 1),
    ([1], [520], 32, 8),
    ([5] * 3, [5, 17, 1044], 4, 4),
    ([1, 0, 2, 17, 3], [31, 40, 33, 48, 16], 8, 2),
    ([1] * 40, [1 + 13 * i for i in range(40)], 5, 1),
    ([9, 1], [777, 16], 24, 2),
    ([33, 70], [33, 200], 3, 3),
    ([130], [300], 16, 2),
    ([2, 1], [5000, 3], 16, 1),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,lengths,H,KV", ATTN)
def test_attention(rows, lengths, H, KV, hd, dtype, causal):
    """Unwritten parts of pages and pages of nobody read as NaN: none may reach an output."""
    from paper_2510_11331_amd import attention_q
    say("attention", rows, lengths, H, KV, hd, dtype, causal)
    r = np.random.default_rng([sum(rows), H, hd])
    c = Case(r, rows, lengths, KV, hd)
    c.fill(r)
    q, q64 = heads(r, c.M, H, hd, dtype)
    got = host(attention_q(q, c.cache(), c.desc, causal))
    close(got, *c.attention(q64, causal), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd,H,KV", [(64, 2, 2), (128, 8, 2), (128, 16, 1)])
@pytest.mark.parametrize("rows,length", [(1, 3000), (5, 12345), (40, 2100)])
def test_attention_finds(rows, length, hd, H, KV, dtype):
    """Every row and head looks for a key of its own: at the ends of pages and of the steps, ranges and tiles that a
    kernel may cut a sequence into.  A lost, doubled or misplaced key is an error of the output's size."""
    from paper_2510_11331_amd import attention_q
    say("finds", rows, length, hd, H, KV, dtype)
    r = np.random.default_rng([rows, length, hd])
    c = Case(r, [rows], [length], KV, hd)
    c.fill(r)
    k, _ = c.pool.get(*c.at(0, np.arange(length)))
    cuts = [0, 15, 16, 31, 32, 63, 64, 127, 128, 255, 256, 511, 512, 1023, 1024, 2047, 2048, length - rows - 1, length - rows]
    at = np.array([cuts[i] if i < len(cuts) else r.integers(0, length - rows + 1) for i in r.permutation(rows * H + 5)[:rows * H]])
    at = at.reshape(rows, H)
    q = 3.0 * k[at, np.arange(H)[None] // (H // KV)] / hd ** 0.5 * 4
    x = t(q.astype(np.float32), dtype)
    want, err = c.attention(host(x))
    got = host(attention_q(x, c.cache(), c.desc))
    close(got, want, err, dtype)
    close(host(attention_q(x, c.cache(), c.desc, causal=False)), *c.attention(host(x), False), dtype)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_nothing(hd, dtype):
    """Sequences of no tokens, negative lengths, rows before the first position: zeros; the others are untouched by it."""
    from paper_2510_11331_amd import attention_q
    say("attention of nothing", hd, dtype)
    r = np.random.default_rng(4)
    c = Case(r, [3, 2, 4, 1], [0, -7, 2, 33], 2, hd)
    c.fill(r)
    q, q64 = heads(r, c.M, 4, hd, dtype)
    for causal in (True, False):
        got = host(attention_q(q, c.cache(), c.desc, causal))
        assert (got[:5] == 0).all() and (not causal or (got[5:7] == 0).all())
        close(got, *c.attention(q64, causal), dtype)


@pytest.mark.parametrize("rows", [6, 100])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_nan(hd, dtype, rows):
    """A NaN key or value reaches the rows that see it, and no others; a value's only its 32 dimensions."""
    from paper_2510_11331_amd import attention_q
    say("attention nan", hd, dtype, rows)
    r = np.random.default_rng(5)
    H, KV, n = 4, 2, 300
    for what, at in (("k", n - 3), ("v", n - 3), ("v", n - rows), ("v", 20), ("k", 70), ("v", n - 1)):
        c = Case(r, [rows, 1], [n, 40], KV, hd)
        c.fill(r)
        x = r.normal(size=(2, 1, KV, hd)).astype(np.float32)
        x["kv".index(what), 0, 1, 3] = np.nan                               # kv head 1, block 0
        c.pool.put(*c.at(0, np.array([at])), x[0], x[1])
        q, q64 = heads(r, c.M, H, hd, dtype)
        got = host(attention_q(q, c.cache(), c.desc))
        want, err = c.attention(q64)
        sees = np.zeros(got.shape, bool)
        sees[:rows][c.pos[:rows] >= at, 2:, :(32 if what == "v" else hd)] = True
        assert np.array_equal(np.isnan(want), sees) and np.array_equal(np.isnan(got), sees)
        close(got[~sees], want[~sees], err[:, ~sees], dtype)
    # infinities and NaN in a query stay in its row and head
    q[2, 1, 0], q[3, 0, 1] = float("nan"), float("inf")
    got = host(attention_q(q, c.cache(), c.desc))
    ok = np.ones(got.shape, bool)
    ok[2, 1] = ok[3, 0] = False
    assert np.isnan(got[2, 1]).all() and np.array_equal(np.isnan(got[ok]), np.isnan(want[ok]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_scales_and_sizes(dtype):
    """Scores far from zero, of both signs and equal; values of many sizes; a scale that is given."""
    from paper_2510_11331_amd import attention_q
    say("attention sizes", dtype)
    r = np.random.default_rng(6)
    hd, H, KV = 128, 4, 2
    for size, scale in ((1e-6, 1e6), (1e4, 1e-4), (30.0, None), (1.0, 0.0), (1.0, -1.0), (1e12, 1e-12)):
        c = Case(r, [4, 3], [100, 650], KV, hd)
        c.fill(r, size * np.exp(3 * r.normal(size=(2, 1, KV, 1))))
        q, q64 = heads(r, c.M, H, hd, dtype)
        if size == 30.0:
            q, q64 = q / 16, q64 / 16
        got = host(attention_q(q, c.cache(), c.desc, scale=scale))
        close(got, *c.attention(q64, scale=scale), dtype)


def test_long_lengths_and_wide_tables():
    """A length far below the table's width, at it, and behind it (NaN); max_len below the length."""
    from paper_2510_11331_amd import KVRows, attention_q
    say("wide tables")
    r = np.random.default_rng(7)
    c = Case(r, [2, 1, 1], [700, 64, 10], 2, 128, width=4096)
    c.fill(r)
    q, q64 = heads(r, c.M, 2, 128, "fp32")
    want, err = c.attention(q64)
    close(host(attention_q(q, c.cache(), c.desc)), want, err, "fp32")
    for max_len in (1, 100, 640, 10 ** 9):
        d = KVRows(c.desc.cu_rows, c.desc.lengths, c.desc.table, max_len)
        close(host(attention_q(q, c.cache(), d)), want, err, "fp32")
    c = Case(r, [2, 1], [64, 64], 2, 128)
    c.fill(r)
    q, q64 = heads(r, 3, 2, 128, "fp32")
    d = KVRows(c.desc.cu_rows, t(np.array([65, 2 ** 31 - 1], dtype=np.int32)), c.desc.table)
    got = host(attention_q(q, c.cache(), d))
    assert np.isfinite(got[0]).all() and np.isnan(got[1:]).all()
    assert np.isnan(host(attention_q(q, c.cache(), d, causal=False))).all()


@pytest.mark.parametrize("KV,hd", [(8, 128), (3, 64)])
def test_pages_past_32_bits(KV, hd):
    """Pages behind 4 GiB of a pool are written, read and attended to."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q
    say("past 32 bits", KV, hd)
    r = np.random.default_rng(8)
    page = KV * 17 * hd
    far = (1 << 32) // page
    cache = KVCacheQ.empty(far + 8, KV, hd)
    assert cache.data.numel() > 1 << 32
    n = 60
    table = np.array([[far + 1, far // 2, far + 7, far + 3], [far // 2 + 1, 0, far, 1]], dtype=np.int32)
    (k, k64), (v, v64) = heads(r, 2 * n, KV, hd, "fp32"), heads(r, 2 * n, KV, hd, "fp32")
    d = KVRows(t(np.array([0, n, 2 * n], dtype=np.int32)), t(np.array([n, n], dtype=np.int32)), t(table))
    kv_append_q(cache, k, v, d)
    got = kv_read_q(cache, d, 2 * n, torch.float32)
    k64, v64 = (kvref.values(*kvref.quantise(x)) for x in (k64, v64))
    assert np.array_equal(host(got[0]), k64) and np.array_equal(host(got[1]), v64)
    q, q64 = heads(r, 2 * n, KV, hd, "fp32")
    got = host(attention_q(q, cache, d))
    for b in range(2):
        s = slice(b * n, b * n + n)
        close(got[s], *kvref.attention(q64[s], k64[s], v64[s], np.tril(np.ones((n, n), bool)), hd ** -0.5), "fp32")


@pytest.mark.parametrize("case", kvplans.CASES, ids=lambda c: c[0])
def test_attention_plans(case):
    """Every kernel, on lengths around its steps and ranges, causal and over all keys; needles among the keys."""
    from paper_2510_11331_amd import attention_q
    name, rows, lengths, H, KV, hd, dtype, width, want_plan = case
    say("plan", name)
    r = np.random.default_rng([H, KV, hd, len(rows)])
    rows = [min(n, m) for n, m in zip(rows, lengths)]
    c = Case(r, rows, lengths, KV, hd, width=width)
    assert kvplans.plan(c.M, H, KV, hd, dtype, len(rows), 16 * width) == want_plan
    c.fill(r)
    q = r.normal(size=(c.M, H, hd))
    for b, m in enumerate(lengths):                      # every other row and head looks for a key of its own
        k, _ = c.pool.get(*c.at(b, np.arange(m)))
        for i in range(c.cu[b], c.cu[b + 1]):
            h = np.arange(i % 2, H, 2)
            q[i, h] = 1.5 * hd ** 0.5 * k[r.integers(0, c.pos[i] + 1, size=len(h)), h // (H // KV)] / (hd / 8)
    x = t(q.astype(np.float32), dtype)
    for causal in (True, False):
        close(host(attention_q(x, c.cache(), c.desc, causal)), *c.attention(host(x), causal), dtype)


@pytest.mark.parametrize("H,KV", [(1, 1), (4, 1), (5, 1), (10, 2), (12, 1), (32, 1), (40, 1)])
@pytest.mark.parametrize("seqs,dtype", [(64, "bf16"), (65, "fp32"), (200, "bf16"), (4096, "bf16"), (4097, "fp32"), (9000, "bf16")])
def test_attention_many_sequences(seqs, dtype, H, KV):
    """A workgroup finds its sequence among all: rows of 0 to 40 in any order, none for whole runs of them.  One token of
    each sequence is cached, so that a row's output is that token's value."""
    from paper_2510_11331_amd import KVRows, KVCacheQ, attention_q, kv_append_q
    import torch
    say("sequences", seqs, dtype, H, KV)
    r = np.random.default_rng([seqs, H])
    hd = 64
    rows = r.choice([0, 0, 1, 1, 1, 1, 2, 3, 5, 17, 40][:11 if seqs < 1000 else 10], size=seqs)
    rows[seqs // 3:seqs // 3 + 30] = 0
    rows[0], rows[-1] = 1, 2
    lengths, table = t(np.ones(seqs, dtype=np.int32)), t(np.arange(seqs, dtype=np.int32)[:, None])
    cache = KVCacheQ(t(np.full((seqs, KV, 17 * hd), 0xff, dtype=np.uint8)))
    x = t(r.integers(-3, 4, size=(seqs, KV, hd)).astype(np.float32), dtype)
    kv_append_q(cache, x, x, KVRows(t(np.arange(seqs + 1, dtype=np.int32)), lengths, table))
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    d = KVRows(t(cu), lengths, table)
    torch.manual_seed(seqs)
    q = torch.randn(int(cu[-1]), H, hd, dtype=dt(dtype), device="cuda")
    want = x[t(np.repeat(np.arange(seqs), rows))].repeat_interleave(H // KV, 1).float()
    # The values are codes; a weight w over the sum w: w, its sum's reciprocal and the product are each rounded to fp32, in
    # bf16 w has 16 bits more, and an integer up to 3 off by 2^-15 of itself rounds to itself.
    slack = want.abs() * (2.0 ** -21 if dtype == "fp32" else 0)
    assert ((attention_q(q, cache, d, False).float() - want).abs() <= slack).all()
    last = torch.zeros(len(q), dtype=torch.bool, device="cuda")
    last[t(cu[1:][rows > 0].astype(np.int64)) - 1] = True
    want *= last[:, None, None]                          # causal: each sequence's last row sees its token, the others nothing
    assert ((attention_q(q, cache, d).float() - want).abs() <= slack).all()


@pytest.mark.parametrize("seqs", [65, 300, 4500])
@pytest.mark.parametrize("rows", [[1], [1, 3], [5, 1, 20, 2, 2], [70, 1]])
@pytest.mark.parametrize("H,KV", [(4, 1), (5, 1), (16, 2), (64, 2)])
def test_attention_few_of_many_sequences(seqs, rows, H, KV):
    """Slots of which most have no rows, at either end and in any order; their keys are split into ranges."""
    from paper_2510_11331_amd import attention_q
    say("few of", seqs, rows, H, KV)
    r = np.random.default_rng([seqs, H, len(rows)])
    for where in ("first", "last", "any"):
        at = {"first": np.arange(len(rows)), "last": seqs - 1 - np.arange(len(rows))[::-1],
              "any": np.sort(r.choice(seqs, size=len(rows), replace=False))}[where]
        n, m = np.zeros(seqs, dtype=int), np.zeros(seqs, dtype=int)
        n[at] = rows
        m[at] = r.integers(100, 700, size=len(rows))
        m[r.integers(0, seqs, size=3)] += 16
        c = Case(r, n.tolist(), m.tolist(), KV, 64, width=400)
        c.fill(r)
        q, q64 = heads(r, c.M, H, 64, "bf16")
        close(host(attention_q(q, c.cache(), c.desc)), *c.attention(q64), "bf16")


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("what", ["large", "small", "tiny", "zero", "nan value", "nan key", "no page", "all sizes"])
def test_attention_shared_values(what, hd):
    """The kernel that shares converted values between its waves: values that its 16-bit form does not hold, NaN and
    pages that are none, in the first steps, in the middle and among the last rows' own keys."""
    from paper_2510_11331_amd import KVRows, attention_q
    say("shared values", what, hd)
    r = np.random.default_rng(12)
    rows, lengths, H, KV = [520, 520], [700, 555], 32, 16
    assert kvplans.plan(sum(rows), H, KV, hd, "bf16", 2, 16 * 44)[0] == 1
    for at in (3, 40, 130, 690):
        c = Case(r, rows, lengths, KV, hd)
        c.fill(r)
        x = r.normal(size=(2, 1, KV, hd)).astype(np.float32)
        table = c.table.copy()
        if what == "large":
            x[1] *= 1e6
        elif what == "small":
            x[1] *= 1e-9
        elif what == "tiny":
            x[1] = 1e-40
        elif what == "zero":
            x[1] = 0
        elif what == "nan value":
            x[1, 0, 3, hd - 1] = np.nan
        elif what == "nan key":
            x[0, 0, 3, 0] = np.inf
        elif what == "all sizes":
            x[1] *= 2.0 ** r.integers(-40, 30, size=(1, KV, 1))
        c.pool.put(*c.at(0, np.array([at])), x[0], x[1])
        q, q64 = heads(r, c.M, H, hd, "bf16")
        want, err = c.attention(q64)
        if what == "no page":
            table[0, at // 16] = -1
            want[:rows[0]][c.pos[:rows[0]] >= at // 16 * 16] = np.nan
        got = host(attention_q(q, c.cache(), KVRows(c.desc.cu_rows, c.desc.lengths, t(table))))
        assert np.array_equal(np.isnan(got), np.isnan(want))
        close(got, want, err, "bf16")


# ------------------------------------------------------------------ as a program runs them


def layer(cache, qkv, d, rope, g, H, KV, hd):
    from paper_2510_11331_amd import attention_q, norm_rope_append_q
    x = qkv.view(-1, H + 2 * KV, hd)
    q = norm_rope_append_q(cache, x[:, :H], x[:, H:H + KV], x[:, H + KV:], d, rope, g, g)
    return attention_q(q, cache, d)


def reference(hist, pos, H, KV, hd, g, cs, dtype):
    """What a layer gives for the last rows of a sequence with the QKV rows hist: keys and values from the whole history."""
    x = hist.reshape(-1, H + 2 * KV, hd)
    n = len(x)
    k = kvref.values(*kvref.quantise(kvref.norm_rope(x[:, H:H + KV], g, cs[:n], 1e-5).astype(np.float32)))
    v = kvref.values(*kvref.quantise(x[:, H + KV:].astype(np.float32)))
    q = kvref.norm_rope(x[pos, :H], g, cs[pos], 1e-5)
    q = host(t(q.astype(np.float32), dtype))
    return kvref.attention(q, k, v, np.arange(n)[None] <= pos[:, None], hd ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decoding(dtype):
    """Prefill of ragged prompts in two chunks, then verification passes of changing numbers of rows with a rollback
    between them, against each sequence's whole history."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, rope_table
    say("decoding", dtype)
    r = np.random.default_rng(9)
    H, KV, hd, B, W = 4, 2, 64, 3, 12
    cache = KVCacheQ(torch.full((B * W, KV, 17 * hd), 255, dtype=torch.uint8, device="cuda"))
    table = t(r.permutation(B * W).reshape(B, W).astype(np.int32))
    rope, g = rope_table(16 * W, hd), t((1 + 0.1 * r.normal(size=hd)).astype(np.float32))
    hist, cs = [np.zeros((0, (H + 2 * KV) * hd)) for _ in range(B)], host(rope)
    for rows, back in (([70, 33, 1], 0), ([40, 0, 90], 0), ([5, 5, 5], 3), ([1, 1, 1], 0), ([2, 0, 1], 0), ([5, 5, 5], 5), ([5, 1, 5], 0)):
        qkv = t(r.normal(size=(sum(rows), (H + 2 * KV) * hd)).astype(np.float32), dtype)
        at = np.concatenate([[0], np.cumsum(rows)])
        for b in range(B):
            hist[b] = np.concatenate([hist[b], host(qkv)[at[b]:at[b + 1]]])
        lengths = np.array([len(h) for h in hist], dtype=np.int32)
        d = KVRows(t(at.astype(np.int32)), t(lengths), table)
        got = host(layer(cache, qkv, d, rope, g, H, KV, hd))
        for b, n in enumerate(rows):
            pos = np.arange(lengths[b] - n, lengths[b])
            want, err = reference(hist[b], pos, H, KV, hd, host(g), cs, dtype)
            close(got[at[b]:at[b + 1]], want, err, dtype)
            hist[b] = hist[b][:len(hist[b]) - min(back, n)]


def test_graph():
    """A captured layer follows lengths, rows, tables and inputs; two graphs and eager calls between their replays."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q, norm_rope, rope_table
    say("graph")
    r = np.random.default_rng(10)
    H, KV, hd, B, W, M = 8, 2, 128, 4, 200, 12
    rope, g = rope_table(16 * W, hd), t((1 + 0.1 * r.normal(size=hd)).astype(np.float32))
    start = torch.from_numpy(kvref.Pool(1, KV, hd).bytes).cuda()
    pages = torch.randint(0, 256, (B * W, KV, 17 * hd), dtype=torch.uint8, device="cuda")
    pages[:, :, 16 * hd:] = 125                                             # any codes, one scale
    graphs = []
    for i in range(2):
        cache = KVCacheQ(pages.clone())
        s = dict(cache=cache, qkv=torch.zeros(M, (H + 2 * KV) * hd, device="cuda"), cu=torch.zeros(B + 1, dtype=torch.int32, device="cuda"),
                 len=torch.zeros(B, dtype=torch.int32, device="cuda"), table=torch.zeros(B, W, dtype=torch.int32, device="cuda"))
        d = KVRows(s["cu"], s["len"], s["table"])

        def run(s=s, d=d):
            o = layer(s["cache"], s["qkv"], d, rope, g, H, KV, hd)
            return o, *kv_read_q(s["cache"], d, M, torch.float32)

        run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s["out"] = run()
        graphs.append((graph, s, d, run))
    for step in range(6):
        for graph, s, d, run in graphs:
            rows = r.multinomial(M - step % 2, np.ones(B) / B)
            lengths = rows + r.integers(0, 16 * W - M, size=B)
            s["qkv"].copy_(t(r.normal(size=(M, (H + 2 * KV) * hd)).astype(np.float32)))
            s["cu"].copy_(t(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)))
            s["len"].copy_(t(lengths.astype(np.int32)))
            s["table"].copy_(t(r.permutation(B * W).reshape(B, W).astype(np.int32)))
        for graph, s, d, run in graphs:
            before = s["cache"].data.clone()
            graph.replay()
            n = int(s["cu"][-1])
            got = [x[:n].clone() for x in s["out"]] + [s["cache"].data.clone()]
            s["cache"].data.copy_(before)
            want = [x[:n] for x in run()] + [s["cache"].data]
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert torch.isfinite(got[0]).all()


def test_streams():
    """Calls on other streams than the current one; two at once on pools of their own."""
    import torch
    from paper_2510_11331_amd import attention_q, kv_append_q, kv_read_q, norm_rope, norm_rope_append_q, rope_table
    say("streams")
    r = np.random.default_rng(11)
    H, KV, hd = 8, 8, 128
    c = Case(r, [5] * 8, [900 + 7 * i for i in range(8)], KV, hd)
    c.fill(r)
    x = t(r.normal(size=(c.M, H + 2 * KV, hd)).astype(np.float32), "bf16")
    q, k, v = x[:, :H], x[:, H:H + KV], x[:, H + KV:]
    g = t(np.ones(hd, dtype=np.float32))
    pos = t(c.pos.astype(np.int32))

    def run(cache, s):
        rope = rope_table(1024, hd, stream=s)
        a = norm_rope(q, k, pos, rope, g, g, stream=s)
        b = norm_rope_append_q(cache, q, k, v, c.desc, rope, g, g, stream=s)
        o = [attention_q(b, cache, c.desc, stream=s)]
        kv_append_q(cache, k, v, c.desc, stream=s)
        o += [attention_q(b, cache, c.desc, stream=s)]
        return [*a, b, *o, *kv_read_q(cache, c.desc, c.M, stream=s)]

    caches = [c.cache() for _ in range(3)]
    want = run(caches[0], None)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, cache in zip(streams, caches[1:]):
            got.append(run(cache, s))
    torch.cuda.synchronize()
    for o in got:
        assert all(torch.equal(a, b) for a, b in zip(o, want))


def test_stream_keeps_memory():
    """Inputs that are dropped while the call's stream has not come to them yet: their memory is not given away."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q, norm_rope, norm_rope_append_q, rope_table
    say("memory on another stream")
    r = np.random.default_rng(12)
    H, KV, hd = 8, 8, 128
    c = Case(r, [9] * 8, [100 + 7 * i for i in range(8)], KV, hd)
    c.fill(r)
    host_x = torch.from_numpy(r.normal(size=(c.M, H + 2 * KV, hd)).astype(np.float32))
    side = torch.cuda.Stream()

    def inputs():
        x = host_x.cuda()
        q, k, v = (y.contiguous() for y in x.split([H, KV, KV], 1))
        d = KVRows(*(y.clone() for y in (c.desc.cu_rows, c.desc.lengths, c.desc.table)))
        return q, k, v, KVCacheQ(c.cache().data.clone()), d, rope_table(1024, hd), torch.ones(hd, device="cuda"), t(c.pos.astype(np.int32))

    def calls(s, q, k, v, cache, d, rope, g, pos):
        a = norm_rope(q, k, pos, rope, g, g, stream=s)
        b = norm_rope_append_q(cache, q, k, v, d, rope, g, g, stream=s)
        o = attention_q(b, cache, d, stream=s)
        kv_append_q(cache, k, v, d, stream=s)
        return [*a, b, o, attention_q(q, cache, d, stream=s), *kv_read_q(cache, d, c.M, stream=s)]

    want = calls(None, *inputs())
    torch.cuda.synchronize()
    for _ in range(3):
        args = inputs()
        sizes = [x.numel() * x.element_size() for x in args[:3]] + [args[3].data.numel()] + [x.numel() * 4 for x in args[5:]]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = calls(side, *args)
        del args
        other = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del other, got


def test_no_rows():
    """Calls without rows or sequences return at once; a pass of more rows than its sequences have leaves the rest."""
    import torch
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q, norm_rope, norm_rope_append_q, rope_table
    say("no rows")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    cache = KVCacheQ(torch.full((3, 2, 17 * 64), 9, dtype=torch.uint8, device="cuda"))
    e, none, some = torch.zeros(0, 2, 64, device="cuda"), KVRows(i32(1), i32(0), i32(0, 1)), KVRows(i32(3), i32(2), i32(2, 4))
    x, rope = torch.full((4, 2, 64), 3.0, device="cuda"), rope_table(8, 64)
    for d in (none, some):
        for y in (e, x):
            assert norm_rope_append_q(cache, y, y, y, d, rope, q_out=y.clone()).eq(y).all()
            kv_append_q(cache, y, y, d)
            assert attention_q(y, cache, d, out=y.clone()).eq(y).all()
            assert all(o.eq(3).all() for o in kv_read_q(cache, d, len(y), torch.float32, y.clone(), y.clone()))
    assert norm_rope(e, e, i32(0), rope)[0].shape == e.shape and rope_table(0, 64).shape == (0, 32, 2)
    assert (cache.data == 9).all()
