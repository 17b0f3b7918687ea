"""Attention over a paged KV cache held in 4 bits, and what writes that cache:
torch tensors in front of libsd's context-free calls (include/sd.h).

A cache (KVCacheQ) is a pool of pages of 16 tokens; keys and values are e2m1
codes with one power-of-two scale per 32 dimensions of a token and head, 17 / 64
of the bytes of a 16-bit cache.  What a pass does is described once for all its
layers (KVRows): which rows belong to which sequence, the sequences' lengths with
these rows, and their pages.  A layer's attention on a QKV product is

    q = norm_rope_append_q(cache, q, k, v, rows, rope, q_gain, k_gain, eps)
    o = attention_q(q, cache, rows)

norm_rope does the norms and the rotation alone, kv_append_q the writing,
kv_read_q gives cached keys and values back.

q, k, v are [rows, heads, head_dim], bfloat16 or float32, head_dim 64 or 128; a
head's entries and a row's heads are adjacent, the rows may lie apart (views of
one QKV product).  Every call enqueues on `stream` (default: the current stream
of the tensors' device) and returns new tensors unless it is given some to write
to; what it uses may be dropped as soon as it returns, as on the current stream.
Arguments that the kernels do not cover raise ValueError, or SDError where
only the library sees it (sizes past its limits, addresses or strides off 16
bytes, eps <= 0, attention on its own queries), before anything is enqueued.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from ._lib import SD_DTYPE_BF16, SD_DTYPE_F32, SD_OK, HeadNorm, KvQPool, KvRows, check, lib
from .ffn_q import _current_device, _elsewhere, _raw_stream

PAGE = 16
_DTYPES = {torch.bfloat16: SD_DTYPE_BF16, torch.float32: SD_DTYPE_F32}


class KVCacheQ:
    """A pool of pages: `data` is uint8 [n_blocks, n_kv_heads, 17 head_dim] on the GPU.  The calls go by its address: the
    fields are read-only."""

    __slots__ = ("_data", "_heads", "_hd", "_index", "_pool", "_at")

    def __init__(self, data: torch.Tensor):
        if data.dim() != 3 or data.dtype != torch.uint8 or not data.is_contiguous() or data.shape[2] not in (17 * 64, 17 * 128):
            raise ValueError("data: contiguous uint8 [n_blocks, n_kv_heads, 17 head_dim], head_dim 64 or 128")
        n, kv, hd = data.shape[0], data.shape[1], data.shape[2] // 17
        if data.numel() == 0 or lib().sd_kv_q_bytes(n, kv, hd) != data.numel():
            raise ValueError(f"no cache of {n} pages of {kv} heads")
        self._data, self._heads, self._hd = data, kv, hd
        self._index = data.get_device()
        self._pool = KvQPool(data.data_ptr(), n, kv, hd)
        self._at = C.addressof(self._pool)

    @classmethod
    def empty(cls, n_blocks: int, n_kv_heads: int, head_dim: int, device="cuda") -> "KVCacheQ":
        """A cache whose pages hold nothing yet: only positions that were written may be read."""
        return cls(torch.empty((n_blocks, n_kv_heads, 17 * head_dim), dtype=torch.uint8, device=device))

    data = property(lambda self: self._data)
    n_blocks = property(lambda self: self._pool.n_blocks)
    n_kv_heads = property(lambda self: self._heads)
    head_dim = property(lambda self: self._hd)


class KVRows:
    """The rows of a pass.  cu_rows [n + 1]: sequence b has the rows cu_rows[b] .. cu_rows[b + 1] - 1; lengths [n]: its
    tokens with these rows, which are its last ones; table [n, width]: the pages of its positions 16 i .. 16 i + 15.  All
    int32 on the GPU, read when a call runs: a captured pass follows what is written to them.  max_len: the longest length
    that the work is to be split for (default: what the table holds, which costs a second launch where that is far more than
    the lengths: 6.3 to 10.9 us for one row on 520 tokens); it may be set between two calls.  The calls go by the tensors'
    addresses: these fields are read-only."""

    __slots__ = ("_cu_rows", "_lengths", "_table", "_max_len", "_index", "_rows", "_at", "_workspace")

    def __init__(self, cu_rows: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, max_len: Optional[int] = None):
        n = lengths.shape[0] if lengths.dim() == 1 else -1
        if n < 0 or cu_rows.shape != (n + 1,) or table.dim() != 2 or table.shape[0] != n or table.shape[1] < 1:
            raise ValueError("cu_rows [n + 1], lengths [n], table [n, width]")
        for t in (cu_rows, lengths, table):
            if t.dtype != torch.int32 or not t.is_contiguous() or t.get_device() != table.get_device():
                raise ValueError("cu_rows, lengths, table: contiguous int32 on one device")
        self._cu_rows, self._lengths, self._table = cu_rows, lengths, table
        self.max_len = max_len
        self._index = table.get_device()
        self._rows = KvRows(cu_rows.data_ptr(), lengths.data_ptr(), table.data_ptr(), n, table.shape[1])
        self._at = C.addressof(self._rows)

    cu_rows = property(lambda self: self._cu_rows)
    lengths = property(lambda self: self._lengths)
    table = property(lambda self: self._table)

    @property
    def max_len(self) -> int:
        return self._max_len

    @max_len.setter
    def max_len(self, n: Optional[int]) -> None:
        if n is not None and n < 1:
            raise ValueError("max_len: at least 1")
        most = 16 * self._table.shape[1]
        self._max_len = min(most, n or most)
        self._workspace = {}                       # bytes of an attention's workspace, by (rows, heads, kv heads, head_dim)


def rope_table(n_pos: int, head_dim: int, theta: float = 10000.0, device="cuda",
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """(cos, sin) of position theta^(-2 i / head_dim): float32 [n_pos, head_dim / 2, 2]."""
    if n_pos < 0 or head_dim not in (64, 128) or not theta > 0:
        raise ValueError("n_pos >= 0, head_dim 64 or 128, theta > 0")
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError("tensors on a GPU are needed")
    index = _current_device() if device.index is None else device.index
    if stream is not None and stream.device.index != index:
        raise ValueError("the stream is of another device than the table")
    if stream is not None or index != _current_device():
        with torch.cuda.device(index) if stream is None else torch.cuda.stream(stream):
            return rope_table(n_pos, head_dim, theta, torch.device("cuda", index))
    out = torch.empty((n_pos, head_dim // 2, 2), dtype=torch.float32, device=torch.device("cuda", index))
    check(lib().sd_rope_table(n_pos, head_dim, theta, out.data_ptr(), _raw_stream(index)), "sd_rope_table")
    return out


def _stride(x: torch.Tensor, what: str, M: int, heads: int, hd: int, dtype: torch.dtype, index: int) -> int:
    """The row stride of heads [M, heads, hd]."""
    if x.shape != (M, heads, hd) or x.dtype != dtype or x.get_device() != index:
        raise ValueError(f"{what}: [{M}, {heads}, {hd}] {dtype} on the device of the others")
    row, head, one = x.stride()
    if M < 2:
        row = heads * hd
        if M == 0:
            return row
    if one != 1 or (head != hd and heads > 1):
        raise ValueError(f"{what}: heads of adjacent entries, adjacent in their row")
    if not heads * hd <= row < 1 << 31:
        raise ValueError(f"{what}: rows apart by at least their length")
    return row


def _norm(hd: int, index: int, rope, q_gain, k_gain, eps: float) -> HeadNorm:
    dt, at = None, [None, None]
    for i, g in enumerate((q_gain, k_gain)):
        if g is not None:
            if g.shape != (hd,) or g.dtype not in _DTYPES or not g.is_contiguous() or g.get_device() != index:
                raise ValueError("gains: contiguous [head_dim], bfloat16 or float32, on the device of q")
            if dt is not None and g.dtype != dt:
                raise ValueError("gains of one type")
            dt, at[i] = g.dtype, g.data_ptr()
    code = SD_DTYPE_BF16 if dt is None else _DTYPES[dt]
    if rope is None:
        return HeadNorm(at[0], at[1], None, code, 0, eps)
    shape = rope.shape
    if (shape[1:] != (hd // 2, 2) or shape[0] < 1 or rope.dtype != torch.float32 or not rope.is_contiguous()
            or rope.get_device() != index):
        raise ValueError("rope: contiguous float32 [positions, head_dim / 2, 2] on the device of q")
    return HeadNorm(at[0], at[1], rope.data_ptr(), code, shape[0], eps)


def _shape(x: torch.Tensor) -> Tuple[int, int, int, int]:
    shape, index = x.shape, x.get_device()
    if len(shape) != 3 or x.dtype not in _DTYPES or shape[2] not in (64, 128) or shape[1] < 1:
        raise ValueError("q, k, v: [rows, heads, head_dim], bfloat16 or float32, head_dim 64 or 128")
    if index < 0:
        raise ValueError("tensors on a GPU are needed")
    return (*shape, index)


def _keep(stream: Optional[torch.cuda.Stream], *tensors: Optional[torch.Tensor]) -> None:
    """Memory that a call on a stream of the caller's choice uses is not given away before the call's work is done."""
    if stream is not None:
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def norm_rope(q: torch.Tensor, k: torch.Tensor, positions: Optional[torch.Tensor] = None, rope: Optional[torch.Tensor] = None,
              q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-5,
              q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(q, k) with every head's RMS norm (gains [head_dim], None: no norm) and then its rotation by (cos, sin) =
    rope[positions[row]] (rope None: no rotation; entries i and i + head_dim / 2 are a pair).  positions int32 [rows].
    q_out, k_out: where they go (the inputs themselves, or memory that overlaps none)."""
    M, H, hd, index = _shape(q)
    if stream is not None or index != _current_device():
        with _elsewhere(q, stream):
            out = norm_rope(q, k, positions, rope, q_gain, k_gain, eps, q_out, k_out)
        _keep(stream, q, k, positions, rope, q_gain, k_gain, q_out, k_out)
        return out
    KV = k.shape[1] if k.dim() == 3 else 0
    if KV < 1 or H % KV:
        raise ValueError("k: [rows, heads, head_dim], its heads a divisor of the query heads")
    ldq, ldk = _stride(q, "q", M, H, hd, q.dtype, index), _stride(k, "k", M, KV, hd, q.dtype, index)
    n = _norm(hd, index, rope, q_gain, k_gain, eps)
    if rope is not None and (positions is None or positions.shape != (M,) or positions.dtype != torch.int32
                             or not positions.is_contiguous() or positions.get_device() != index):
        raise ValueError("positions: contiguous int32 [rows] on the device of q")
    ldqo, ldko = H * hd, KV * hd
    if q_out is None:
        q_out = torch.empty(M, H, hd, dtype=q.dtype, device=q.device)
    else:
        ldqo = _stride(q_out, "q_out", M, H, hd, q.dtype, index)
    if k_out is None:
        k_out = torch.empty(M, KV, hd, dtype=q.dtype, device=q.device)
    else:
        ldko = _stride(k_out, "k_out", M, KV, hd, q.dtype, index)
    rc = lib().sd_norm_rope(M, H, KV, hd, _DTYPES[q.dtype], q.data_ptr(), ldq, k.data_ptr(), ldk,
                            None if rope is None else positions.data_ptr(), C.addressof(n), q_out.data_ptr(), ldqo,
                            k_out.data_ptr(), ldko, _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_norm_rope")
    return q_out, k_out


def _same_device(cache: KVCacheQ, rows: KVRows, index: int) -> None:
    if cache._index != index or rows._index != index:
        raise ValueError("cache, rows and tensors on one device")


def kv_append_q(cache: KVCacheQ, k: torch.Tensor, v: torch.Tensor, rows: KVRows,
                stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantise the rows' keys and values into the cache, at their positions."""
    M, KV, hd, index = _shape(k)
    if stream is not None or index != _current_device():
        with _elsewhere(k, stream):
            kv_append_q(cache, k, v, rows)
        return _keep(stream, k, v, cache._data, rows._cu_rows, rows._lengths, rows._table)
    if KV != cache._heads or hd != cache._hd:
        raise ValueError(f"k: [rows, {cache._heads}, {cache._hd}]")
    _same_device(cache, rows, index)
    ldk, ldv = _stride(k, "k", M, KV, hd, k.dtype, index), _stride(v, "v", M, KV, hd, k.dtype, index)
    rc = lib().sd_kv_append_q(cache._at, rows._at, M, _DTYPES[k.dtype], k.data_ptr(), ldk, v.data_ptr(), ldv, _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_kv_append_q")


def norm_rope_append_q(cache: KVCacheQ, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rows: KVRows,
                       rope: Optional[torch.Tensor] = None, q_gain: Optional[torch.Tensor] = None,
                       k_gain: Optional[torch.Tensor] = None, eps: float = 1e-5, q_out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """norm_rope at the rows' positions: q is returned, k (its values in float32) and v go into the cache.  q_out: where
    q goes (q itself, or memory that overlaps no input)."""
    M, H, hd, index = _shape(q)
    if stream is not None or index != _current_device():
        with _elsewhere(q, stream):
            out = norm_rope_append_q(cache, q, k, v, rows, rope, q_gain, k_gain, eps, q_out)
        _keep(stream, q, k, v, rope, q_gain, k_gain, q_out, cache._data, rows._cu_rows, rows._lengths, rows._table)
        return out
    KV = cache._heads
    if hd != cache._hd or H % KV:
        raise ValueError(f"q: heads of {cache._hd}, a multiple of {KV}")
    _same_device(cache, rows, index)
    ldq = _stride(q, "q", M, H, hd, q.dtype, index)
    ldk, ldv = _stride(k, "k", M, KV, hd, q.dtype, index), _stride(v, "v", M, KV, hd, q.dtype, index)
    n = _norm(hd, index, rope, q_gain, k_gain, eps)
    ldqo = H * hd
    if q_out is None:
        q_out = torch.empty(M, H, hd, dtype=q.dtype, device=q.device)
    else:
        ldqo = _stride(q_out, "q_out", M, H, hd, q.dtype, index)
    rc = lib().sd_norm_rope_append_q(cache._at, rows._at, M, H, _DTYPES[q.dtype], q.data_ptr(), ldq, k.data_ptr(), ldk,
                                     v.data_ptr(), ldv, C.addressof(n), q_out.data_ptr(), ldqo, _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_norm_rope_append_q")
    return q_out


def kv_read_q(cache: KVCacheQ, rows: KVRows, n_rows: int, dtype: torch.dtype = torch.bfloat16,
              k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(k, v) [n_rows, heads, head_dim] of dtype at the rows' positions.  k_out, v_out: where they go."""
    index = cache._index
    if index < 0:
        raise ValueError("a cache on a GPU is needed")
    if stream is not None or index != _current_device():
        with _elsewhere(cache._data, stream):
            out = kv_read_q(cache, rows, n_rows, dtype, k_out, v_out)
        _keep(stream, k_out, v_out, cache._data, rows._cu_rows, rows._lengths, rows._table)
        return out
    KV, hd = cache._heads, cache._hd
    if dtype not in _DTYPES or n_rows < 0:
        raise ValueError("at least 0 rows, bfloat16 or float32")
    _same_device(cache, rows, index)
    ldk = ldv = KV * hd
    if k_out is None:
        k_out = torch.empty(n_rows, KV, hd, dtype=dtype, device=cache._data.device)
    else:
        ldk = _stride(k_out, "k_out", n_rows, KV, hd, dtype, index)
    if v_out is None:
        v_out = torch.empty(n_rows, KV, hd, dtype=dtype, device=cache._data.device)
    else:
        ldv = _stride(v_out, "v_out", n_rows, KV, hd, dtype, index)
    rc = lib().sd_kv_read_q(cache._at, rows._at, n_rows, _DTYPES[dtype], k_out.data_ptr(), ldk, v_out.data_ptr(), ldv,
                            _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_kv_read_q")
    return k_out, v_out


def attention_q(q: torch.Tensor, cache: KVCacheQ, rows: KVRows, causal: bool = True, scale: Optional[float] = None,
                out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """softmax(scale q K^T) V [rows, heads, head_dim] over the cached positions up to the row's own (causal) or all of its
    sequence's; scale: head_dim^-0.5 unless given.  Query heads share kv heads in runs.  out: where it goes (memory that
    overlaps no input; on q is refused)."""
    M, H, hd, index = _shape(q)
    if stream is not None or index != _current_device():
        with _elsewhere(q, stream):
            given, out = out, attention_q(q, cache, rows, causal, scale, out)
        _keep(stream, q, given, cache._data, rows._cu_rows, rows._lengths, rows._table)
        return out
    KV = cache._heads
    if hd != cache._hd or H % KV:
        raise ValueError(f"q: heads of {cache._hd}, a multiple of {KV}")
    _same_device(cache, rows, index)
    ldq, ldo = _stride(q, "q", M, H, hd, q.dtype, index), H * hd
    if out is None:
        out = torch.empty(M, H, hd, dtype=q.dtype, device=q.device)
    else:
        ldo = _stride(out, "out", M, H, hd, q.dtype, index)
    L = lib()
    sizes = (M, H, KV, hd)
    ws = rows._workspace.get(sizes)
    if ws is None:
        ws = rows._workspace[sizes] = L.sd_attention_q_workspace_bytes(M, H, KV, hd, rows._rows.n_seqs, rows._max_len)
    work = torch.empty(ws, dtype=torch.uint8, device=q.device) if ws else None
    rc = L.sd_attention_q(cache._at, rows._at, M, H, _DTYPES[q.dtype], q.data_ptr(), ldq, out.data_ptr(), ldo, causal,
                          hd ** -0.5 if scale is None else scale, rows._max_len, work.data_ptr() if ws else None, ws,
                          _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_attention_q")
    return out
