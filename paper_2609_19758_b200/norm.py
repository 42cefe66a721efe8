"""Residual addition and RMS norm on the accumulator of a verified output projection (``include/fpsk_decoder.h``), with the backward
pass and an 8-bit output.

Argument marshalling only, like ``attention.py``: every step runs inside the CUDA library, asynchronously on the given (or the
current) stream of the tensors' device.  Outputs and workspaces are the caller's tensors; wrong shapes, types, devices or strides
raise ValueError or TypeError, what the library refuses raises FpskError.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import attention as A
from . import fpsk
from .fpsk import ERR_SHAPE, FpskError


def add_rms_norm(x: torch.Tensor, residual: Optional[torch.Tensor], weight: Optional[torch.Tensor], y: torch.Tensor,
                 residual_out: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, group: int = 0, eps: float = 1e-6,
                 status: Optional[torch.Tensor] = None, stream=None) -> None:
    """h = x + residual (tokens, dim), stored to residual_out (which may be residual); y = h rsqrt(mean(h^2) + eps) weight, rounded once.
    A float8_e4m3fn y holds y / scale, with scale (tokens, groups) filled for each `group` channels (32, 64, 128 or 256; 0: the row)."""
    b = A._binding or A._bind()
    A._check(b.add_rms_norm(x, residual, weight, y, residual_out, scale, group, eps, status, A._stream(b.device(x), stream)), "fpsk_add_rms_norm")


def add_rms_norm_workspace(dim: int, device=None) -> torch.Tensor:
    """Workspace of add_rms_norm_backward for rows of dim channels; serves one call at a time."""
    A._bind()
    n = int(fpsk.lib().fpsk_add_norm_workspace_bytes(dim))
    if n == 0:
        raise FpskError(ERR_SHAPE, "fpsk_add_norm_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device="cuda" if device is None else device)


def add_rms_norm_backward(h: torch.Tensor, dy: torch.Tensor, weight: Optional[torch.Tensor], dx: torch.Tensor,
                          dweight: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None,
                          eps: float = 1e-6, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward pass of add_rms_norm from the sum h: dx (the type of dy), the gradient of x and of the residual alike, from dy and from
    dh, what arrives at the sum through the residual stream; and the FP32 gradient of the weight (overwritten; it needs ws)."""
    b = A._binding or A._bind()
    A._check(b.add_rms_norm_backward(h, dy, weight, dx, dweight, ws, dh, eps, status, A._stream(b.device(h), stream)), "fpsk_add_rms_norm_backward")


class AddRMSNorm(torch.autograd.Function):
    """add_rms_norm with its gradients for autograd: ``apply(x, residual, weight, out_dtype, eps)`` returns y in out_dtype (16 bits or FP32: an
    8-bit y, which wants scales, is add_rms_norm's alone) and the sum h in the residual's type (in x's where residual is None).  The
    gradient is computed and rounded once in the type of x where all types agree, else in FP32; a second derivative is refused."""

    @staticmethod
    def forward(ctx, x, residual, weight, out_dtype, eps):
        ctx.set_materialize_grads(False)
        y = torch.empty(x.shape, dtype=out_dtype, device=x.device)
        h = torch.empty(x.shape, dtype=x.dtype if residual is None else residual.dtype, device=x.device)
        add_rms_norm(x, residual, weight, y, residual_out=h, eps=eps)
        ctx.save_for_backward(h, weight)
        ctx.more = (x.dtype, None if residual is None else residual.dtype, out_dtype, eps)
        return y, h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dh):
        h, weight = ctx.saved_tensors
        x_dtype, residual_dtype, out_dtype, eps = ctx.more
        grad_dtype = out_dtype if x_dtype == out_dtype == h.dtype else torch.float32
        if dy is None:
            dy = torch.zeros(h.shape, dtype=grad_dtype, device=h.device)
        dy, dh = ((g if g.stride(-1) == 1 or g.shape[-1] == 1 else g.contiguous()).to(grad_dtype) if g is not None else None for g in (dy, dh))
        dx = torch.empty(h.shape, dtype=grad_dtype, device=h.device)
        dw, ws = None, None
        if weight is not None and ctx.needs_input_grad[2]:
            dw, ws = torch.empty(weight.shape, dtype=torch.float32, device=weight.device), add_rms_norm_workspace(h.shape[1], h.device)
        add_rms_norm_backward(h, dy, weight, dx, dw, ws, dh=dh, eps=eps)
        return (dx.to(x_dtype), None if residual_dtype is None else dx.to(residual_dtype), None if dw is None else dw.to(weight.dtype), None, None)
