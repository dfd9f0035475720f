"""Matrices in the microscaled 4-bit format (MXFP4) and the products of them.

Thin plumbing over the ``saem_mx_*`` calls: device memory and arguments here, arithmetic in
libsaem's kernels.  Everything is enqueued on the current stream unless a stream (or its handle) is given; a result that
is allocated in such a call belongs to that stream, as if it were the current one.
"""
from __future__ import annotations

import contextlib
from typing import Optional

import torch

from . import binding as B
from .build import host_calls

_calls = host_calls()
_DTYPE = {torch.float32: B.SAEM_OUT_F32, torch.bfloat16: B.SAEM_OUT_BF16}


def _dtype(t: torch.Tensor) -> int:
    try:
        return _DTYPE[t.dtype]
    except KeyError:
        raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "float32 or bfloat16 wanted, not %s" % t.dtype) from None


def _matrix(t: torch.Tensor, what: str, rows: Optional[int] = None, cols: Optional[int] = None) -> int:
    """The row stride of a matrix on the GPU whose columns are consecutive (and whose shape is [rows, cols], if given)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or not t.is_cuda or (stride[1] != 1 and shape[1] > 1):
        raise B.SaemError(B.SAEM_ERR_INVALID_ARG, what + ": a matrix on the GPU with consecutive columns is wanted")
    if rows is not None and shape != (rows, cols):
        raise B.SaemError(B.SAEM_ERR_SHAPE, what)
    return stride[0]


def _allocated_on(stream):
    """A context whose allocations belong to `stream` (None: the current stream).  Memory out of the current stream's pool may
    still be in use by earlier work there, which the call's stream does not wait for."""
    if stream is None:
        return contextlib.nullcontext()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    return torch.cuda.stream(stream)


class MxTensor:
    """A quantised matrix [rows, cols]: `codes` and `scales` as include/saem.h describes them (uint8)."""

    __slots__ = ("rows", "cols", "codes", "scales")

    def __init__(self, rows: int, cols: int, codes: torch.Tensor, scales: torch.Tensor):
        for t, size in ((codes, B.saem_mx_codes_bytes(rows, cols)), (scales, B.saem_mx_scales_bytes(rows, cols))):
            if t.dtype != torch.uint8 or not t.is_contiguous() or t.numel() < size or (rows and not size):
                raise B.SaemError(B.SAEM_ERR_SHAPE, "MxTensor")
        self.rows, self.cols, self.codes, self.scales = rows, cols, codes, scales

    @property
    def device(self):
        return self.codes.device

    def nbytes(self) -> int:
        return self.codes.numel() + self.scales.numel()


def empty(rows: int, cols: int, device="cuda") -> MxTensor:
    """An MxTensor whose contents are unspecified."""
    return MxTensor(rows, cols, torch.empty(B.saem_mx_codes_bytes(rows, cols), dtype=torch.uint8, device=device),
                    torch.empty(B.saem_mx_scales_bytes(rows, cols), dtype=torch.uint8, device=device))


def quantize(x: torch.Tensor, out: Optional[MxTensor] = None, stream=None) -> MxTensor:
    """x [rows, cols] float32 or bfloat16 to the microscaled format."""
    if out is None:
        _dtype(x), _matrix(x, "quantize")
        with _allocated_on(stream):
            out = empty(x.shape[0], x.shape[1], x.device)
    code = _calls.quantize(x, out.rows, out.cols, out.codes, out.scales, stream)
    if code:
        raise B.SaemError(code, "quantize")
    return out


def dequantize(q: MxTensor, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.float32, stream=None) -> torch.Tensor:
    """The values a quantised matrix stands for, as float32 or bfloat16 (exact in both)."""
    if out is None:
        with _allocated_on(stream):
            out = torch.empty(q.rows, q.cols, dtype=dtype, device=q.device)
    code = _calls.dequantize(q.codes, q.scales, q.rows, q.cols, out, stream)
    if code:
        raise B.SaemError(code, "dequantize")
    return out


def matmul(a: MxTensor, w: MxTensor, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
           status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """out[m, n] = sum_k a[m, k] * w[n, k], float32 sums, bfloat16 or float32 out."""
    if a.cols != w.cols:
        raise B.SaemError(B.SAEM_ERR_SHAPE, "matmul")
    if out is None:
        with _allocated_on(stream):
            out = torch.empty(a.rows, w.rows, dtype=dtype, device=a.device)
    code = _calls.matmul(a.codes, a.scales, a.rows, w.codes, w.scales, w.rows, w.cols, out, status, stream)
    if code:
        raise B.SaemError(code, "matmul")
    return out


class Linear:
    """A projection whose weights are quantised once and whose activations are quantised in every call.

    `max_rows` sizes the workspace; calls of one Linear must be ordered on the GPU (they share it), and after the stream that
    was current when it was made."""

    def __init__(self, weight: MxTensor, max_rows: int):
        if not (weight.codes.is_cuda and weight.codes.device == weight.scales.device):
            raise B.SaemError(B.SAEM_ERR_INVALID_ARG, "Linear: weights on one GPU are wanted")
        self.weight, self.max_rows = weight, max_rows
        self.workspace = torch.empty(max(256, B.saem_mx_linear_workspace_bytes(max_rows, weight.cols)), dtype=torch.uint8,
                                     device=weight.device)
        self.workspace[:4].zero_()

    def __call__(self, x: torch.Tensor, out: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
                 stream=None) -> torch.Tensor:
        """x [m, k] float32 or bfloat16 -> [m, n]."""
        w = self.weight
        if out is None:
            with _allocated_on(stream):
                out = torch.empty(x.shape[0], w.rows, dtype=dtype, device=x.device)
        code = _calls.linear(x, w.codes, w.scales, w.rows, w.cols, out, self.workspace, self.max_rows, stream)
        if code:
            raise B.SaemError(code, "Linear")
        return out

    def device_status(self) -> int:
        """The status word of the calls so far, whatever their streams (synchronises the device); 0 unless a device-side wait ran
        out.  Clears it."""
        torch.cuda.synchronize(self.workspace.device)
        code = int(self.workspace[:4].view(torch.int32).item())
        if code:
            self.workspace[:4].zero_()
            torch.cuda.synchronize(self.workspace.device)
        return code
