"""What the 4-bit cache's calls do with memory, without a GPU: where it is taken from, and what may follow a call."""
import contextlib
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
needs_lib = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2510_11331_amd", "libsd.so")), reason="libsd.so not built")


@needs_lib
@pytest.mark.parametrize("where", ["stream", "device", "here"])
def test_rope_table_takes_memory_on_its_stream(where, monkeypatch):
    """The table's memory is of the stream that writes it: taken of another one, it may still be in use there, or be given
    away there before it is written."""
    from paper_2510_11331_amd import kv_q
    inside, seen = [], []

    @contextlib.contextmanager
    def context():
        inside.append(where)
        yield
        inside.pop()

    class Lib:
        @staticmethod
        def sd_rope_table(n_pos, head_dim, theta, out, stream):
            seen.append(("write", list(inside)))
            return 0

    empty = torch.empty

    def take(*a, **k):
        seen.append(("take", list(inside)))
        return empty(*a, **{**k, "device": "cpu"})

    monkeypatch.setattr(kv_q, "lib", lambda: Lib)
    monkeypatch.setattr(kv_q, "_elsewhere", lambda t, stream: None if inside or where == "here" else context())
    monkeypatch.setattr(kv_q, "_raw_stream", lambda index: None)
    monkeypatch.setattr(torch, "empty", take)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: context())
    monkeypatch.setattr(torch.cuda, "device", lambda d: context())
    monkeypatch.setattr(kv_q, "_current_device", lambda: 1 if where == "device" and not inside else 0)
    given = type("Stream", (), {"device": torch.device("cuda", 0)})() if where == "stream" else None
    out = kv_q.rope_table(4, 64, device="cuda:0", stream=given)
    assert out.shape == (4, 32, 2)
    want = [] if where == "here" else [where]
    assert seen == [("take", want), ("write", want)]


def rows_of(width, max_len=None):
    from paper_2510_11331_amd import KVRows
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    return KVRows(i32(2), i32(1), i32(1, width), max_len)


@needs_lib
def test_max_len_between_calls(monkeypatch):
    """max_len may be set between two calls: each gets the workspace that its own max_len needs."""
    from paper_2510_11331_amd import KVCacheQ, _lib, kv_q
    real, seen = _lib.lib(), []
    cache, rows = KVCacheQ(torch.zeros(4, 8, 17 * 128, dtype=torch.uint8)), rows_of(2048, 500)

    class Lib:
        sd_attention_q_workspace_bytes = real.sd_attention_q_workspace_bytes

        @staticmethod
        def sd_attention_q(pool, rows, M, H, dtype, q, ldq, out, ldo, causal, scale, max_len, work, size, stream):
            seen.append((max_len, size))
            return _lib.SD_OK if size >= real.sd_attention_q_workspace_bytes(M, H, 8, 128, 1, max_len) else _lib.SD_EINVAL

    monkeypatch.setattr(kv_q, "lib", lambda: Lib)
    monkeypatch.setattr(kv_q, "_raw_stream", lambda index: None)
    monkeypatch.setattr(kv_q, "_current_device", lambda: -1)
    monkeypatch.setattr(kv_q, "_shape", lambda x: (*x.shape, -1))          # (host tensors stand for the GPU's)
    q = torch.zeros(1, 32, 128, dtype=torch.bfloat16)
    for n, given in ((500, 500), (32768, 32768), (16, 16), (32768, 10 ** 6), (1, 1), (32768, None), (16000, 16000)):
        if (n, given) != (500, 500):
            rows.max_len = given
        assert rows.max_len == n
        kv_q.attention_q(q, cache, rows)
        assert seen[-1] == (n, real.sd_attention_q_workspace_bytes(1, 32, 8, 128, 1, n))
    for bad in (0, -1):
        with pytest.raises(ValueError):
            rows.max_len = bad
    assert rows.max_len == 16000


@needs_lib
def test_tensors_of_handles_stay():
    """The calls read addresses taken when a handle was made: its tensors and sizes cannot be exchanged."""
    from paper_2510_11331_amd import KVCacheQ
    cache, rows = KVCacheQ(torch.zeros(4, 2, 17 * 64, dtype=torch.uint8)), rows_of(3)
    for handle, names in ((cache, ("data", "n_blocks", "n_kv_heads", "head_dim")), (rows, ("cu_rows", "lengths", "table"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(handle, name, getattr(handle, name))


@needs_lib
def test_workspace_grows_with_max_len():
    """A workspace for a length is enough for every shorter one, and so for a call whose table ends before max_len."""
    from paper_2510_11331_amd import _lib
    need = _lib.lib().sd_attention_q_workspace_bytes
    lengths = [1, 16, 255, 256, 1000, 1535, 1536, 2048, 2559, 2560, 4000, 8191, 8192, 14336, 20000, 33000, 70000, 131072, 10 ** 6, 1 << 24]
    for hd in (64, 128):
        for B in (1, 2, 3, 4, 5, 7, 8, 12, 16, 31, 33, 36, 48, 64, 65, 200, 1000):
            for n in (1, 2, 3, 5, 9, 17, 40, 130, 700):
                for H, KV in ((1, 1), (8, 1), (8, 8), (17, 1), (20, 5), (40, 5), (32, 8), (32, 32), (64, 8)):
                    sizes = [need(B * n, H, KV, hd, B, x) for x in lengths]
                    assert sizes == sorted(sizes), (hd, B, n, H, KV, sizes)


@needs_lib
def test_attention_refuses_outputs_on_its_queries():
    """Other workgroups may still read a query when an output is written: also partly on it, or between its rows.  (The
    pointers are never dereferenced.)"""
    import ctypes as C
    from paper_2510_11331_amd import _lib
    L, A = _lib.lib(), 1 << 24
    pool, rows = _lib.KvQPool(1 << 20, 9, 2, 64), _lib.KvRows(1 << 20, 1 << 20, 1 << 20, 2, 3)
    row = 4 * 64 * 2                                                        # bytes of a row of 4 heads in bf16

    def refused(M, out, ldq=4 * 64, ldo=4 * 64):
        return L.sd_attention_q(C.addressof(pool), C.addressof(rows), M, 4, _lib.SD_DTYPE_BF16, A, ldq, A + out, ldo, 1, 0.1, 48,
                                1 << 20, 1 << 20, None) == _lib.SD_EINVAL

    for M in (1, 2, 7):
        for at in (0, 16, row - 16, (M - 1) * row, M * row - 16, -16, 16 - row, 16 - M * row):
            assert refused(M, at), (M, at)
    wide = 8 * 64                                                           # rows with as much between them
    for M in (2, 7):
        for at in (0, 16, row - 16, row + 16, 2 * row, 2 * row - 16, -16, -row + 16, -row - 16, -2 * row, (M - 1) * 2 * row):
            assert refused(M, at, wide, wide), (M, at)
        # of other strides: the output's second row on the query's third, its last row on the query's first
        assert refused(5, 4 * row - 3 * row, wide, 3 * 4 * 64) and refused(5, -4 * 3 * row, wide, 3 * 4 * 64)
        assert refused(3, -2 * row, 4 * 64, 4 * 64)


@needs_lib
@pytest.mark.skipif(torch.cuda.is_available(), reason="the call that is not refused would run")
def test_attention_refusals_with_outputs_apart():
    """Each argument that is refused, in a call that is not refused without it (which then finds no GPU)."""
    import ctypes as C
    from paper_2510_11331_amd import _lib
    L, E, A = _lib.lib(), _lib.SD_EINVAL, 1 << 20
    pool = dict(data=A, n_blocks=3000, n_kv_heads=8, head_dim=128)
    rows = dict(cu_rows=A, lengths=A, table=A, n_seqs=1, table_width=2048)
    n = L.sd_attention_q_workspace_bytes(5, 32, 8, 128, 1, 32768)
    assert n > 0
    good = dict(M=5, H=32, dtype=_lib.SD_DTYPE_BF16, q=A, ldq=4096, out=2 * A, ldo=4096, causal=1, scale=0.1, max_len=0, ws=4 * A, n=n)

    def call(p={}, r={}, **a):
        keep = _lib.KvQPool(*{**pool, **p}.values()), _lib.KvRows(*{**rows, **r}.values())
        return L.sd_attention_q(C.addressof(keep[0]), C.addressof(keep[1]), *{**good, **a}.values(), None)

    for fine in ({}, dict(out=A + 5 * 4096 * 2), dict(out=A - 5 * 4096 * 2), dict(ldq=8192, out=A + 4096 * 2, ldo=8192), dict(max_len=1000, ws=None, n=0)):
        assert call(**fine) not in (E, _lib.SD_OK), fine
    for bad in (dict(M=-1), dict(M=(1 << 20) + 1), dict(H=0), dict(H=33), dict(H=1032), dict(dtype=2), dict(q=None), dict(q=A + 8), dict(ldq=4088),
                dict(ldq=4100), dict(out=None), dict(out=2 * A + 8), dict(ldo=4088), dict(ldo=4100), dict(max_len=-1), dict(ws=None),
                dict(ws=4 * A + 8), dict(n=n - 1), dict(n=0)):
        assert call(**bad) == E, bad
    for bad in (dict(data=None), dict(data=A + 8), dict(n_blocks=0), dict(n_kv_heads=0), dict(head_dim=96)):
        assert call(p=bad) == E, bad
    for bad in (dict(cu_rows=None), dict(lengths=A + 1), dict(table=None), dict(n_seqs=-1), dict(table_width=0), dict(table_width=(1 << 20) + 1)):
        assert call(r=bad) == E, bad
    assert call(M=0, q=None) == call(r=dict(n_seqs=0)) == _lib.SD_OK


@needs_lib
def test_longest_max_len():
    """A max_len that no table reaches is as good as one that a table does: the same plan, and a workspace that is enough."""
    import ctypes as C
    from paper_2510_11331_amd import _lib
    L = _lib.lib()
    for hd in (64, 128):
        for B in (1, 2, 4, 8, 16, 36, 64):
            for n in (1, 5, 17):
                for H, KV in ((1, 1), (8, 1), (20, 5), (32, 8), (40, 5)):
                    plans = []
                    for x in (1 << 24, 2 ** 31 - 31, 2 ** 31 - 1):
                        assert L.sd_attention_q_workspace_bytes(B * n, H, KV, hd, B, x) == L.sd_attention_q_workspace_bytes(B * n, H, KV, hd, B, 1 << 24)
                        p = _lib.AttentionQPlan()
                        assert L.sd_plan_attention_q(B * n, H, KV, hd, B, x, 0, C.byref(p)) == _lib.SD_OK
                        plans.append((p.shared, p.vectors, p.waves, p.key_ranges, p.streamed))
                    assert plans[1] == plans[0] and plans[2] == plans[0]
