"""The feed-forward network in 8-bit floating point: torch tensors in front of
libsd's context-free 8-bit calls (include/sd.h).

Rows of 8-bit numbers are a pair (q, exps): e4m3 codes float8_e4m3fn [M, K8], K8
= K rounded up to a multiple of 128, and one power-of-two scale per 128 entries,
float8_e8m0fnu [M, Ke], Ke = K8 / 128 rounded up to a multiple of 4.  A layer's
feed-forward pass on a residual stream x is

    x, q, e = add_rmsnorm_q(x, gain, eps, add=attention_output)
    q, e = gate_up_q(q, e, w_gate_up)
    x = linear_q(q, e, w_down, add=x)

Sums are as exact as fp32 ones.  fast=True: of more than 64 rows they run on the 8-bit
matrix instruction, which takes about half the time and drops low bits of the products
that it adds (sd_linear_q_fast).

Every call enqueues on `stream` (default: the current stream of the tensors'
device) and returns new tensors unless it is given some to write to.  Arguments
that the kernels do not cover raise ValueError, or SDError where only the
library sees it (sizes past its limits, addresses off their alignment, eps <= 0),
before anything is enqueued.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from ._lib import SD_DTYPE_BF16, SD_DTYPE_F32, SD_OK, check, lib

BLOCK = 128
_DTYPES = {torch.bfloat16: SD_DTYPE_BF16, torch.float32: SD_DTYPE_F32}
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# of the current device and its current stream; a few tenths of a microsecond that short calls notice
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _k8(K: int) -> int:
    return (K + 127) & ~127


def _ke(K: int) -> int:
    return (K + 511) // 512 * 4


def _elsewhere(t: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    """None if a call on t and stream is one on the current device and stream, else the context in which it is."""
    index = t.get_device()
    if index < 0:
        raise ValueError("tensors on a GPU are needed")
    if stream is None:
        return None if index == _current_device() else torch.cuda.device(index)
    if stream.device != t.device:
        raise ValueError("the stream is of another device than the tensors")
    return torch.cuda.stream(stream)


class LinearQ:
    """A packed weight [N, K] (y = x W^T): `data` holds sd_linear_q_bytes(N, K) bytes on the GPU."""

    __slots__ = ("data", "N", "K")

    def __init__(self, data: torch.Tensor, N: int, K: int):
        n = lib().sd_linear_q_bytes(N, K)
        if n == 0:
            raise ValueError(f"no packed matrix of {N} x {K}")
        if data.dtype != torch.uint8 or data.shape != (n,) or not data.is_contiguous():
            raise ValueError(f"a packed {N} x {K} matrix is a contiguous uint8 tensor of {n} entries")
        self.data, self.N, self.K = data, N, K

    @property
    def codes(self) -> torch.Tensor:
        """The code tiles, in packed order."""
        return self.data[:(self.N + 15) // 16 * 16 * _k8(self.K)].view(_E4M3)

    @property
    def exps(self) -> torch.Tensor:
        """The scales [ceil(N / 128), Ke]."""
        return self.data[(self.N + 15) // 16 * 16 * _k8(self.K):].view(_E8M0).view(-1, _ke(self.K))


def pack_linear_q(w: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> LinearQ:
    """Quantise and pack a weight [N, K] (bfloat16 or float32)."""
    if w.dim() != 2 or w.dtype not in _DTYPES or not w.is_contiguous():
        raise ValueError("w: contiguous [N, K], bfloat16 or float32")
    N, K = w.shape
    n = lib().sd_linear_q_bytes(N, K)
    if n == 0:
        raise ValueError(f"no packed matrix of {N} x {K}")
    there = _elsewhere(w, stream)
    if there is not None:
        with there:
            return pack_linear_q(w)
    data = torch.empty(n, dtype=torch.uint8, device=w.device)
    check(lib().sd_pack_linear_q(w.data_ptr(), data.data_ptr(), N, K, _DTYPES[w.dtype], _raw_stream(w.get_device())),
          "sd_pack_linear_q")
    return LinearQ(data, N, K)


def add_rmsnorm_q(x: torch.Tensor, gain: torch.Tensor, eps: float, add: Optional[torch.Tensor] = None,
                  x_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                  ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(s, q, exps) with s = x + add and q, exps the rows of s / sqrt(mean(s^2) + eps) * gain.  x [M, d] is bfloat16 or
    float32; add of its type [M, d], or [n, M, d] (n <= 6, all of them are added), or None (s is then x itself).  gain [d]
    is bfloat16 or float32.  x_out: where s goes (x itself, or memory that overlaps no input)."""
    there = _elsewhere(x, stream) if x.is_cuda else None
    if there is not None:
        with there:
            return add_rmsnorm_q(x, gain, eps, add, x_out)
    t, dev, index = x.dtype, x.device, x.get_device()
    if x.dim() != 2 or t not in _DTYPES or not x.is_contiguous():
        raise ValueError("x: contiguous [M, d], bfloat16 or float32")
    M, d = x.shape
    if not 1 <= d <= 16384:
        raise ValueError("rows of 1 to 16384 entries")
    if gain.shape != (d,) or gain.dtype not in _DTYPES or not gain.is_contiguous() or gain.get_device() != index:
        raise ValueError("gain: [d], bfloat16 or float32, on the device of x")
    n = 0
    if add is not None:
        n = 1 if add.dim() == 2 else add.shape[0]
        if (add.dim() not in (2, 3) or add.shape[-2:] != x.shape or add.dtype != t or not add.is_contiguous()
                or add.get_device() != index):
            raise ValueError("add: contiguous [M, d] or [n, M, d] of x's type and device")
        if n > 6:
            raise ValueError("at most 6 addends")
    if x_out is not None:
        if n and (x_out.shape != x.shape or x_out.dtype != t or not x_out.is_contiguous() or x_out.get_device() != index):
            raise ValueError("x_out: as x")
        if not n and x_out.data_ptr() != x.data_ptr():
            raise ValueError("x_out is written with addends only")
    if index < 0:
        raise ValueError("tensors on a GPU are needed")
    out = x if not n else torch.empty_like(x) if x_out is None else x_out
    q = torch.empty((M, _k8(d)), dtype=_E4M3, device=dev)
    exps = torch.empty((M, _ke(d)), dtype=_E8M0, device=dev)
    rc = lib().sd_add_rmsnorm_q(M, d, _DTYPES[t], x.data_ptr(), n, add.data_ptr() if n else None, out.data_ptr(),
                                gain.data_ptr(), _DTYPES[gain.dtype], eps, q.data_ptr(), exps.data_ptr(), _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_add_rmsnorm_q")
    return out, q, exps


def _rows(q: torch.Tensor, exps: torch.Tensor, w: LinearQ) -> int:
    M, K = q.shape[0] if q.dim() else 0, w.K
    if q.dtype != _E4M3 or q.shape != (M, _k8(K)) or not q.is_contiguous():
        raise ValueError(f"q: contiguous float8_e4m3fn [M, {_k8(K)}]")
    if exps.dtype != _E8M0 or exps.shape != (M, _ke(K)) or not exps.is_contiguous():
        raise ValueError(f"exps: contiguous float8_e8m0fnu [M, {_ke(K)}]")
    if not q.get_device() == exps.get_device() == w.data.get_device():
        raise ValueError("rows and weight on one device")
    return M


def linear_q(q: torch.Tensor, exps: torch.Tensor, w: LinearQ, add: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32,
             stream: Optional[torch.cuda.Stream] = None, fast: bool = False) -> torch.Tensor:
    """[add +] rows W^T as [M, N] of dtype (float32 or bfloat16).  out: where it goes (rows may lie apart); add: float32
    with out's strides, or out itself."""
    there = _elsewhere(q, stream) if q.is_cuda else None
    if there is not None:
        with there:
            return linear_q(q, exps, w, add, out, dtype, None, fast)
    M, N, index = _rows(q, exps, w), w.N, q.get_device()
    ldo = N
    if out is not None:
        dtype = out.dtype
        if (out.shape != (M, N) or out.get_device() != index or not (N == 1 or M == 0 or out.stride(1) == 1)
                or not (M <= 1 or N <= out.stride(0) < 1 << 31)):
            raise ValueError("out: [M, N] with adjacent columns, on the device of the rows")
        if M > 1:
            ldo = out.stride(0)
    if dtype not in _DTYPES:
        raise ValueError("outputs are float32 or bfloat16")
    if add is not None and (add.dtype != torch.float32 or add.shape != (M, N) or add.get_device() != index
                            or not (N == 1 or M == 0 or add.stride(1) == 1) or not (M <= 1 or add.stride(0) == ldo)):
        raise ValueError("add: float32 [M, N] with the strides of the output")
    if index < 0:
        raise ValueError("tensors on a GPU are needed")
    L = lib()
    ws = L.sd_linear_q_workspace_bytes(M, N, w.K)
    if out is None:
        out = torch.empty((M, N), dtype=dtype, device=q.device)
    work = torch.empty(ws, dtype=torch.uint8, device=q.device) if ws else None
    call = L.sd_linear_q_fast if fast else L.sd_linear_q
    rc = call(M, N, w.K, q.data_ptr(), exps.data_ptr(), w.data.data_ptr(),
              None if add is None else add.data_ptr(), out.data_ptr(), ldo, _DTYPES[dtype],
              work.data_ptr() if ws else None, ws, _raw_stream(index))
    if rc != SD_OK:
        check(rc, "sd_linear_q")
    return out


def gate_up_q(q: torch.Tensor, exps: torch.Tensor, w: LinearQ, stream: Optional[torch.cuda.Stream] = None,
              fast: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows (q, exps) of silu(gate) * up, w the packed [2 F, K] with gate and up rows interleaved in blocks of 16
    (engine.interleave_gate_up)."""
    there = _elsewhere(q, stream) if q.is_cuda else None
    if there is not None:
        with there:
            return gate_up_q(q, exps, w, None, fast)
    M, F, dev = _rows(q, exps, w), w.N // 2, q.device
    L = lib()
    if w.N % 32 or F > 1 << 18:
        raise ValueError("gate and up rows come in blocks of 16, at most 2^18 of each")
    if not q.is_cuda:
        raise ValueError("tensors on a GPU are needed")
    q_out = torch.empty((M, _k8(F)), dtype=_E4M3, device=dev)
    exps_out = torch.empty((M, _ke(F)), dtype=_E8M0, device=dev)
    ws = L.sd_gate_up_q_workspace_bytes(M, F, w.K)
    work = torch.empty(ws, dtype=torch.uint8, device=dev) if ws else None
    call = L.sd_gate_up_q_fast if fast else L.sd_gate_up_q
    rc = call(M, F, w.K, q.data_ptr(), exps.data_ptr(), w.data.data_ptr(), q_out.data_ptr(),
              exps_out.data_ptr(), work.data_ptr() if ws else None, ws, _raw_stream(q.get_device()))
    if rc != SD_OK:
        check(rc, "sd_gate_up_q")
    return q_out, exps_out
