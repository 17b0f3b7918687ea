"""The feed-forward network in 8-bit floating point: torch tensors in front of
libsd's context-free 8-bit calls (include/sd.h).

Rows of 8-bit numbers are a pair (q, exps): e4m3 codes float8_e4m3fn [M, K8], K8
= K rounded up to a multiple of 128, and one power-of-two scale per 128 entries,
float8_e8m0fnu [M, Ke], Ke = K8 / 128 rounded up to a multiple of 4.  A layer's
feed-forward pass on a residual stream x is

    x, q, e = add_rmsnorm_q(x, gain, eps, add=attention_output)
    q, e = gate_up_q(q, e, w_gate_up)
    x = linear_q(q, e, w_down, add=x)

Every call enqueues on `stream` (default: the current stream of the tensors'
device) and returns new tensors unless it is given some to write to.  Arguments
that the kernels do not cover raise ValueError before anything is enqueued.
"""
from __future__ import annotations

from contextlib import nullcontext
from typing import Optional, Tuple

import torch

from ._lib import SD_DTYPE_BF16, SD_DTYPE_F32, SD_OK, check, lib

BLOCK = 128
_DTYPES = {torch.bfloat16: SD_DTYPE_BF16, torch.float32: SD_DTYPE_F32}
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _k8(K: int) -> int:
    return (K + 127) & ~127


def _ke(K: int) -> int:
    return (K + 511) // 512 * 4


class _On:
    """The device and stream of a call: tensors are made and work is enqueued there."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        _need(device.type == "cuda", "tensors on a GPU are needed")
        if stream is not None:
            _need(stream.device == device, "the stream is of another device than the tensors")
            self.ctx = torch.cuda.stream(stream)
        else:
            self.ctx = nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)
        self.device = device

    def __enter__(self) -> int:
        self.ctx.__enter__()
        return torch.cuda.current_stream(self.device).cuda_stream

    def __exit__(self, *a):
        return self.ctx.__exit__(*a)


class LinearQ:
    """A packed weight [N, K] (y = x W^T): `data` holds sd_linear_q_bytes(N, K) bytes on the GPU."""

    __slots__ = ("data", "N", "K")

    def __init__(self, data: torch.Tensor, N: int, K: int):
        n = lib().sd_linear_q_bytes(N, K)
        _need(n > 0, f"no packed matrix of {N} x {K}")
        _need(data.dtype == torch.uint8 and data.dim() == 1 and data.numel() == n and data.is_contiguous(),
              f"a packed {N} x {K} matrix is a contiguous uint8 tensor of {n} entries")
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
    _need(w.dim() == 2 and w.dtype in _DTYPES and w.is_contiguous(), "w: contiguous [N, K], bfloat16 or float32")
    N, K = w.shape
    n = lib().sd_linear_q_bytes(N, K)
    _need(n > 0, f"no packed matrix of {N} x {K}")
    with _On(w.device, stream) as s:
        data = torch.empty(n, dtype=torch.uint8, device=w.device)
        check(lib().sd_pack_linear_q(w.data_ptr(), data.data_ptr(), N, K, _DTYPES[w.dtype], s), "sd_pack_linear_q")
    return LinearQ(data, N, K)


def add_rmsnorm_q(x: torch.Tensor, gain: torch.Tensor, eps: float, add: Optional[torch.Tensor] = None,
                  x_out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                  ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(s, q, exps) with s = x + add and q, exps the rows of s / sqrt(mean(s^2) + eps) * gain.  x [M, d] is bfloat16 or
    float32; add of its type [M, d], or [n, M, d] (n <= 6, all of them are added), or None (s is then x itself).  gain [d]
    is bfloat16 or float32.  x_out: where s goes (may be x)."""
    _need(x.dim() == 2 and x.dtype in _DTYPES and x.is_contiguous(), "x: contiguous [M, d], bfloat16 or float32")
    M, d = x.shape
    _need(1 <= d <= 16384, "rows of 1 to 16384 entries")
    _need(gain.shape == (d,) and gain.dtype in _DTYPES and gain.is_contiguous() and gain.device == x.device,
          "gain: [d], bfloat16 or float32, on the device of x")
    n = 0
    if add is not None:
        n = 1 if add.dim() == 2 else add.shape[0]
        _need(add.shape[-2:] == x.shape and add.dim() in (2, 3) and add.dtype == x.dtype and add.is_contiguous()
              and add.device == x.device, "add: contiguous [M, d] or [n, M, d] of x's type and device")
        _need(n <= 6, "at most 6 addends")
    if n:
        _need(x_out is None or (x_out.shape == x.shape and x_out.dtype == x.dtype and x_out.is_contiguous()
                                and x_out.device == x.device), "x_out: as x")
    else:
        _need(x_out is None or x_out.data_ptr() == x.data_ptr(), "x_out is written with addends only")
    with _On(x.device, stream) as s:
        out = x if not n else torch.empty_like(x) if x_out is None else x_out
        q = torch.empty(M, _k8(d), dtype=_E4M3, device=x.device)
        exps = torch.empty(M, _ke(d), dtype=_E8M0, device=x.device)
        rc = lib().sd_add_rmsnorm_q(M, d, _DTYPES[x.dtype], x.data_ptr(), n, add.data_ptr() if n else None,
                                    out.data_ptr(), gain.data_ptr(), _DTYPES[gain.dtype], eps, q.data_ptr(),
                                    exps.data_ptr(), s)
    if rc != SD_OK:
        check(rc, "sd_add_rmsnorm_q")
    return out, q, exps


def _rows(q: torch.Tensor, exps: torch.Tensor, w: LinearQ) -> int:
    K = w.K
    _need(q.dtype == _E4M3 and q.dim() == 2 and q.shape[1] == _k8(K) and q.is_contiguous(),
          f"q: contiguous float8_e4m3fn [M, {_k8(K)}]")
    M = q.shape[0]
    _need(exps.dtype == _E8M0 and exps.shape == (M, _ke(K)) and exps.is_contiguous(),
          f"exps: contiguous float8_e8m0fnu [M, {_ke(K)}]")
    _need(q.device == exps.device == w.data.device, "rows and weight on one device")
    return M


def linear_q(q: torch.Tensor, exps: torch.Tensor, w: LinearQ, add: Optional[torch.Tensor] = None,
             out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32,
             stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """[add +] rows W^T as [M, N] of dtype (float32 or bfloat16).  out: where it goes (rows may lie apart); add: float32
    with out's strides, or out itself."""
    M, N = _rows(q, exps, w), w.N
    if out is not None:
        dtype = out.dtype
        _need(out.shape == (M, N) and (N == 1 or M == 0 or out.stride(1) == 1) and (M <= 1 or out.stride(0) >= N)
              and out.device == q.device, "out: [M, N] with adjacent columns, on the device of the rows")
    _need(dtype in _DTYPES, "outputs are float32 or bfloat16")
    ldo = out.stride(0) if out is not None and M > 1 else N
    _need(ldo < 1 << 31, "rows of out less than 2^31 entries apart")
    if add is not None:
        _need(add.dtype == torch.float32 and add.shape == (M, N) and add.device == q.device
              and (N == 1 or M == 0 or add.stride(1) == 1) and (M <= 1 or add.stride(0) == ldo),
              "add: float32 [M, N] with the strides of the output")
    with _On(q.device, stream) as s:
        if out is None:
            out = torch.empty(M, N, dtype=dtype, device=q.device)
        ws = lib().sd_linear_q_workspace_bytes(M, N, w.K)
        work = torch.empty(ws, dtype=torch.uint8, device=q.device)
        rc = lib().sd_linear_q(M, N, w.K, q.data_ptr(), exps.data_ptr(), w.data.data_ptr(),
                               None if add is None else add.data_ptr(), out.data_ptr(), ldo, _DTYPES[dtype],
                               work.data_ptr(), ws, s)
    if rc != SD_OK:
        check(rc, "sd_linear_q")
    return out


def gate_up_q(q: torch.Tensor, exps: torch.Tensor, w: LinearQ, stream: Optional[torch.cuda.Stream] = None
              ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Rows (q, exps) of silu(gate) * up, w the packed [2 F, K] with gate and up rows interleaved in blocks of 16
    (engine.interleave_gate_up)."""
    M, F = _rows(q, exps, w), w.N // 2
    ws = lib().sd_gate_up_q_workspace_bytes(M, F, w.K) if w.N % 32 == 0 else 0
    _need(ws > 0, "gate and up rows come in blocks of 16, at most 2^18 of each")
    with _On(q.device, stream) as s:
        q_out = torch.empty(M, _k8(F), dtype=_E4M3, device=q.device)
        exps_out = torch.empty(M, _ke(F), dtype=_E8M0, device=q.device)
        work = torch.empty(ws, dtype=torch.uint8, device=q.device)
        rc = lib().sd_gate_up_q(M, F, w.K, q.data_ptr(), exps.data_ptr(), w.data.data_ptr(), q_out.data_ptr(),
                                exps_out.data_ptr(), work.data_ptr(), ws, s)
    if rc != SD_OK:
        check(rc, "sd_gate_up_q")
    return q_out, exps_out
