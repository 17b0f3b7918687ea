"""The 4-bit cache without a GPU: the format's reference, sizes, and what the calls refuse before anything is enqueued."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import kvref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
needs_lib = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2510_11331_amd", "libsd.so")), reason="libsd.so not built")


def test_codes():
    """Every code's number, the ties, the scale's border; a block's number is within half a step of its value."""
    v = np.array([0, 0.25, 0.26, 0.74, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 6.0])
    assert kvref.code(v).tolist() == [0, 0, 1, 1, 2, 2, 4, 4, 6, 6, 7, 7] and kvref.code(-v).tolist() == [8, 8, 9, 9, 10, 10, 12, 12, 14, 14, 15, 15]
    assert np.array_equal(kvref.code(kvref.number(np.arange(16, dtype=np.uint8))), np.arange(16))
    assert kvref.exponent(np.array([0.0, 2.0 ** -149, 6 * 2.0 ** -126, 6.0001 * 2.0 ** -126, 6.0, 6.0001, 3.0, 3.4e38])).tolist() == \
        [1, 1, 1, 2, 127, 128, 126, 253]
    x = np.random.default_rng(0).normal(size=(50, 64)) * np.exp(np.random.default_rng(1).normal(size=(50, 1)))
    c, E = kvref.quantise(x)
    step = 2.0 ** (np.repeat(E, 32, -1) - 127.0)
    assert (np.abs(kvref.values(c, E) - x) <= step * np.where(np.abs(x) < 2 * step, 0.25, np.where(np.abs(x) < 4 * step, 0.5, 1.0))).all()
    x[3, 40] = np.inf
    c, E = kvref.quantise(x)
    assert E[3].tolist()[1] == 255 and np.isnan(kvref.values(c, E)[3, 32:]).all() and np.isfinite(kvref.values(c, E)[3, :32]).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_page_layout(hd):
    """A page's bytes are each used once."""
    p = kvref.Pool(1, 1, hd)
    assert sorted(np.concatenate([x.reshape(-1) for x in (p.kc, p.vc, p.ks, p.vs)]).tolist()) == list(range(17 * hd))


@needs_lib
def test_sizes():
    from paper_2510_11331_amd import _lib
    L = _lib.lib()
    assert L.sd_kv_q_bytes(5, 3, 64) == 5 * 3 * 17 * 64 and L.sd_kv_q_bytes(1 << 24, 8, 128) == (1 << 24) * 8 * 17 * 128
    for bad in ((0, 1, 64), ((1 << 24) + 1, 1, 64), (1, 0, 64), (1, 1025, 64), (1, 1, 96), (1, 1, 0), (-1, 1, 64)):
        assert L.sd_kv_q_bytes(*bad) == 0, bad
    for bad in ((0, 8, 8, 64, 1, 100), (1, 0, 8, 64, 1, 100), (1, 9, 8, 64, 1, 100), (1, 8, 8, 32, 1, 100), (1, 8, 8, 64, 0, 100),
                (1, 8, 8, 64, 1, 0), ((1 << 20) + 1, 8, 8, 64, 1, 100), (1, 8, 8, 64, (1 << 20) + 1, 100)):
        assert L.sd_attention_q_workspace_bytes(*bad) == 0, bad


@needs_lib
def test_calls_refuse():
    """The pointers are never dereferenced."""
    from paper_2510_11331_amd import _lib
    L, E, OK, A = _lib.lib(), _lib.SD_EINVAL, _lib.SD_OK, 1 << 20
    BF, F32 = _lib.SD_DTYPE_BF16, _lib.SD_DTYPE_F32
    pool = dict(data=A, n_blocks=9, n_kv_heads=4, head_dim=64)
    rows = dict(cu_rows=A, lengths=A, table=A, n_seqs=2, table_width=3)
    norm = dict(q_gain=A, k_gain=A, rope=A, gain_dtype=BF, n_pos=10, eps=1e-5)

    def call(f, args, p=pool, r=rows, n=norm):
        keep = _lib.KvQPool(*p.values()), _lib.KvRows(*r.values()), _lib.HeadNorm(*n.values())
        at = {"pool": keep[0], "rows": keep[1], "norm": keep[2]}
        return f(*[C.addressof(at[v]) if isinstance(v, str) else v for v in args.values()], None)

    def check(f, args, bad, empty):
        for b in bad:
            assert call(f, {**args, **b}) == E, (f.__name__, b)
        for b in empty:
            assert call(f, {**args, **b}) == OK, (f.__name__, b)
        if "pool" in args:
            for b in (dict(data=None), dict(data=A + 8), dict(n_blocks=0), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=32),
                      dict(n_blocks=(1 << 24) + 1)):
                assert call(f, args, p={**pool, **b}) == E, (f.__name__, b)
            for b in (dict(cu_rows=None), dict(lengths=None), dict(table=None), dict(cu_rows=A + 2), dict(n_seqs=-1), dict(table_width=0),
                      dict(n_seqs=(1 << 20) + 1), dict(table_width=(1 << 20) + 1)):
                assert call(f, args, r={**rows, **b}) == E, (f.__name__, b)
            assert call(f, args, r={**rows, "n_seqs": 0, "cu_rows": None}) == OK
            assert call(f, {**args, "pool": None}) == E and call(f, {**args, "rows": None}) == E
        if "norm" in args:
            for b in (dict(gain_dtype=2), dict(n_pos=0), dict(n_pos=(1 << 24) + 1), dict(eps=0.0), dict(eps=float("nan")), dict(rope=A + 8),
                      dict(q_gain=A + 1), dict(k_gain=A + 1), dict(k_gain=A + 2, gain_dtype=F32)):
                assert call(f, args, n={**norm, **b}) == E, (f.__name__, b)
            assert call(f, {**args, "norm": None}) == E

    big = (1 << 20) + 1
    heads = lambda x, ld: [{x: None}, {x: A + 8}, {ld: 4 * 64 - 8}, {ld: 4 * 64 + 4}]
    ap = dict(pool="pool", rows="rows", M=5, dtype=BF, k=A, ldk=256, v=A, ldv=256)
    check(L.sd_kv_append_q, ap, [dict(M=-1), dict(M=big), dict(dtype=2), *heads("k", "ldk"), *heads("v", "ldv")], [dict(M=0, k=None)])
    check(L.sd_kv_read_q, ap, [dict(M=-1), dict(M=big), dict(dtype=-1), *heads("k", "ldk"), *heads("v", "ldv")], [dict(M=0, v=None)])
    nr = dict(M=5, H=4, KV=4, hd=64, dtype=BF, q=A, ldq=256, k=A, ldk=256, pos=A, norm="norm", q_out=A, ldqo=256, k_out=A, ldko=256)
    check(L.sd_norm_rope, nr, [dict(M=-1), dict(M=big), dict(H=0), dict(H=6), dict(KV=0), dict(H=2048, KV=1024), dict(hd=32), dict(dtype=2),
                               dict(pos=None), dict(pos=A + 2), *heads("q", "ldq"), *heads("k", "ldk"), *heads("q_out", "ldqo"),
                               *heads("k_out", "ldko")], [dict(M=0, q=None)])
    both = dict(pool="pool", rows="rows", M=5, H=4, dtype=F32, q=A, ldq=256, k=A, ldk=256, v=A, ldv=256, norm="norm", q_out=A, ldqo=256)
    check(L.sd_norm_rope_append_q, both, [dict(M=-1), dict(H=0), dict(H=5), dict(dtype=2), *heads("q", "ldq")[:3], *heads("k", "ldk")[:3],
                                          *heads("v", "ldv")[:3], *heads("q_out", "ldqo")[:3], dict(ldq=257)], [dict(M=0, q=None)])
    n = max(L.sd_attention_q_workspace_bytes(5, 4, 4, 64, 2, 48), 1)
    at = dict(pool="pool", rows="rows", M=5, H=4, dtype=BF, q=A, ldq=256, out=A, ldo=256, causal=1, scale=0.125, max_len=48, ws=A, n=n)
    check(L.sd_attention_q, at, [dict(M=-1), dict(M=big), dict(H=0), dict(H=6), dict(dtype=2), dict(max_len=-1), *heads("q", "ldq"),
                                 *heads("out", "ldo")], [dict(M=0, q=None)])
    # grids that no launch has
    wide, M = dict(pool, n_kv_heads=1024), 1 << 20
    for f, a in ((L.sd_kv_append_q, ap), (L.sd_kv_read_q, ap), (L.sd_norm_rope_append_q, {**both, "H": 1024}), (L.sd_attention_q, {**at, "H": 1024})):
        assert call(f, {k: 65536 if k[:2] == "ld" else v for k, v in {**a, "M": M}.items()}, p=wide, r=dict(rows, n_seqs=M)) == E, f.__name__
    assert call(L.sd_norm_rope, {**nr, "M": M, "H": 1024, "KV": 1024, **dict.fromkeys(("ldq", "ldk", "ldqo", "ldko"), 65536)}) == E
    assert L.sd_plan_attention_q(M, 1024, 1024, 64, M, 16, BF, C.byref(_lib.AttentionQPlan())) == E
    assert L.sd_rope_table(0, 64, 1e4, None, None) == OK
    for bad in ((-1, 64, 1e4, A), (4, 32, 1e4, A), (4, 64, 0.0, A), (4, 64, float("nan"), A), (4, 64, 1e4, None), (4, 64, 1e4, A + 8),
                ((1 << 24) + 1, 64, 1e4, A)):
        assert L.sd_rope_table(*bad, None) == E, bad


@needs_lib
def test_python_refuses():
    """Shapes, types and layouts (host tensors: none of these calls gets as far as needing a GPU)."""
    from paper_2510_11331_amd import KVCacheQ, KVRows, attention_q, kv_append_q, kv_read_q, norm_rope, norm_rope_append_q, rope_table

    def refused(f, *a, **k):
        with pytest.raises(ValueError):
            f(*a, **k)

    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    for bad in (u8(4, 2, 17 * 96), u8(4, 17 * 64), u8(0, 2, 17 * 64), u8(4, 1025, 17 * 64), u8(4, 2, 34 * 64)[:, :, ::2], u8(4, 2, 17 * 64).int()):
        refused(KVCacheQ, bad)
    cache = KVCacheQ(u8(4, 2, 17 * 64))
    assert (cache.n_blocks, cache.n_kv_heads, cache.head_dim) == (4, 2, 64)
    for bad in ((i32(3), i32(3), i32(3, 4)), (i32(4), i32(3), i32(2, 4)), (i32(4), i32(3), i32(3, 0)), (i32(4).long(), i32(3), i32(3, 4)),
                (i32(4), i32(3), i32(4, 3).t()), (i32(4), i32(3, 1), i32(3, 4)), (i32(4), i32(6)[::2], i32(3, 4))):
        refused(KVRows, *bad)
    refused(KVRows, i32(4), i32(3), i32(3, 4), 0)
    rows = KVRows(i32(4), i32(3), i32(3, 4))
    assert rows.max_len == 64 and KVRows(i32(4), i32(3), i32(3, 4), 7).max_len == 7
    x = torch.zeros(3, 2, 64)
    for y in (x, x.half(), torch.zeros(3, 2, 96), torch.zeros(3, 128), torch.zeros(3, 0, 64)):       # host tensors, and worse
        refused(attention_q, y, cache, rows)
        refused(kv_append_q, cache, y, y, rows)
        refused(norm_rope, y, y)
        refused(norm_rope_append_q, cache, y, y, y, rows)
    refused(kv_read_q, cache, rows, 3)
    refused(rope_table, -1, 64, device="cpu")
    refused(rope_table, 4, 96, device="cpu")
    refused(rope_table, 4, 64, 0.0, device="cpu")
    refused(rope_table, 4, 64, device="cpu")


@needs_lib
def test_row_strides():
    """What the wrappers take as rows of heads."""
    from paper_2510_11331_amd.kv_q import _stride
    f = torch.float32
    x = torch.zeros(5, 10, 64)
    assert _stride(x, "x", 5, 10, 64, f, -1) == 640 and _stride(x[:, 2:5], "x", 5, 3, 64, f, -1) == 640
    assert _stride(x[:1, 2:5], "x", 1, 3, 64, f, -1) == 192 and _stride(x[:0], "x", 0, 10, 64, f, -1) == 640
    assert _stride(x[:, 3:4], "x", 5, 1, 64, f, -1) == 640
    for y in (x[:, ::2], x[:, :, :32], x.expand(5, 10, 64).transpose(0, 1), x.double(), x[:1].expand(5, 10, 64)):
        with pytest.raises(ValueError):
            _stride(y, "y", *y.shape[:2], 64, f, -1)


@needs_lib
def test_plans():
    """The GPU cases run on the kernels that they name, and there is no kernel that none of them runs on."""
    import kvplans
    seen = set()
    for name, rows, lengths, H, KV, hd, dtype, width, want in kvplans.CASES:
        got = kvplans.plan(sum(rows), H, KV, hd, dtype, len(rows), 16 * width)
        assert got == want, (name, got)
        seen.add(kvplans.kind(got, hd, dtype))
    parts = lambda k: (k[:6], (k[0], k[1], k[6]))             # the first kernel, and the second
    first, second = {parts(k)[0] for k in seen}, {parts(k)[1] for k in seen}
    missing = {}
    for hd in (64, 128):
        for dtype in ("bf16", "fp32"):
            for B in (1, 2, 7, 16, 33, 64, 200):
                for n in (1, 2, 5, 17, 100, 700, 2048):
                    for H, KV in ((1, 1), (8, 1), (40, 5), (32, 8), (32, 32), (64, 8), (128, 128), (640, 64)):
                        if B * n * H > 1 << 27:                   # (past a grid's threads)
                            continue
                        for length in (16, 500, 1500, 1600, 3000, 9000, 33000, 400000):
                            k = kvplans.kind(kvplans.plan(B * n, H, KV, hd, dtype, B, length), hd, dtype)
                            for part, have in zip(parts(k), (first, second)):
                                if part not in have:
                                    missing.setdefault(part, (B, n, H, KV, length))
    assert not missing


@needs_lib
def test_workspace():
    """Key ranges need it, whole and aligned."""
    from paper_2510_11331_amd import _lib
    L, E, A = _lib.lib(), _lib.SD_EINVAL, 1 << 20
    pool, rows = _lib.KvQPool(A, 3000, 8, 128), _lib.KvRows(A, A, A, 1, 2048)
    n = L.sd_attention_q_workspace_bytes(1, 32, 8, 128, 1, 32768)
    assert n >= 32 * 2 * (128 + 2) * 4 and L.sd_attention_q_workspace_bytes(1, 32, 8, 128, 1, 1000) == 0
    call = lambda ws, size, max_len: L.sd_attention_q(C.addressof(pool), C.addressof(rows), 1, 32, 0, A, 4096, A, 4096, 1, 0.1, max_len, ws,
                                                      size, None)
    assert call(None, n, 0) == call(A, n - 4, 0) == call(A + 4, n, 0) == call(None, 0, 10 ** 6) == E
    p = _lib.AttentionQPlan()
    for bad in ((0, 8, 8, 64, 1, 100, 0), (1, 9, 8, 64, 1, 100, 0), (1, 8, 8, 64, 0, 100, 0), (1, 8, 8, 64, 1, 0, 0), (1, 8, 8, 64, 1, 100, 2)):
        assert L.sd_plan_attention_q(*bad, C.byref(p)) == E, bad
    assert L.sd_plan_attention_q(1, 8, 8, 64, 1, 100, 0, None) == E
