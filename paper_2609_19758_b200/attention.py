"""The attention operators that follow a verified projection (``include/fpsk_attention.h``): norms and rotation of
queries and keys with their backward pass, writes to a paged cache, and attention of new tokens over it.

Argument marshalling only, like ``fpsk.py``, in C++ (``csrc/binding.cpp``): every step runs inside the CUDA library,
asynchronously on the given (or the current) stream of the tensors' device.  Outputs and workspaces are the caller's tensors; wrong shapes, types,
devices or strides raise ValueError or TypeError, what the library refuses raises FpskError.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import build, fpsk
from .fpsk import ERR_SHAPE, STATUS_OK, FpskError

_binding = None


def _bind():
    """The C++ binding, given the functions of the library that this process has loaded."""
    global _binding
    if _binding is None:
        if not os.path.exists(BINDING_PATH):
            raise FileNotFoundError(f"{BINDING_PATH} is missing: build it with `python -m paper_2609_19758_b200.build`")
        if not build.binding_is_current():
            raise RuntimeError(f"{BINDING_PATH} is not made for {build.binding_mark()} build it again with `python -m paper_2609_19758_b200.build`")
        from . import _binding as b
        L = fpsk.lib()
        vp, sz = C.c_void_p, C.c_size_t
        for name, restype, argtypes in (("fpsk_norm_rope_workspace_bytes", sz, [C.c_int32]), ("fpsk_paged_attention_workspace_bytes", sz, []),
                                        ("fpsk_attention_workspace_init", C.c_int, [vp, sz, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
        b.bind(*(C.cast(getattr(L, n), vp).value for n in ("fpsk_qk_norm_rope", "fpsk_qk_norm_rope_backward", "fpsk_paged_append",
                                                           "fpsk_paged_attention")))
        _binding = b
    return _binding


BINDING_PATH = build.BINDING


def _check(rc: int, where: str) -> None:
    if rc != STATUS_OK:
        raise FpskError(rc, where)


def _stream(device: int, stream) -> int:
    """The given stream, else the current one of the device."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device)


def _workspace(nbytes, device, stream) -> torch.Tensor:
    """A workspace of nbytes() bytes on the device (None: the current one)."""
    with torch.cuda.device(device):
        n = nbytes()
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        _check(fpsk.lib().fpsk_attention_workspace_init(ws.data_ptr(), n, _stream(ws.get_device(), stream)), "fpsk_attention_workspace_init")
    return ws


def rotary_tables(n_pos: int, rot_dim: int, base: float = 10000.0, device=None):
    """cos and sin of pos * base^(-2 i / rot_dim), FP32 (n_pos, rot_dim / 2), from 64-bit angles."""
    inv = base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device or "cuda") / max(rot_dim, 1))
    a = torch.arange(n_pos, dtype=torch.float64, device=inv.device)[:, None] * inv
    return a.cos().float(), a.sin().float()


def qk_norm_rope(q: Optional[torch.Tensor], k: Optional[torch.Tensor], cos, sin, positions, q_out, k_out, q_weight=None,
                 k_weight=None, eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """q (tokens, query heads, dim) and k (tokens, key heads, dim), any strides with contiguous channels (views into the
    projection's accumulator): z = x rsqrt(mean(x^2) + eps) w for each head where a weight is given, rotated by the token's
    position, rounded once into q_out and k_out.  Either of q and k may be None."""
    b = _binding or _bind()
    _check(b.qk_norm_rope(q, k, cos, sin, positions, q_out, k_out, q_weight, k_weight, eps, interleaved, status,
                          _stream(b.device(q if q is not None else k), stream)), "fpsk_qk_norm_rope")


def norm_rope_workspace(head_dim: int, device=None, stream=None) -> torch.Tensor:
    """Workspace of qk_norm_rope_backward; serves one call at a time."""
    _bind()
    n = int(fpsk.lib().fpsk_norm_rope_workspace_bytes(head_dim))
    if n == 0:
        raise FpskError(ERR_SHAPE, "fpsk_norm_rope_workspace_bytes")
    return _workspace(lambda: n, device, stream)


def qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dq_weight, dk_weight, ws: torch.Tensor,
                          q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                          status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward pass of qk_norm_rope from its inputs q, k and the gradients of its outputs: fills dq, dk (the type of dq_out)
    and the FP32 gradients of the weights (overwritten)."""
    b = _binding or _bind()
    _check(b.qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dq_weight, dk_weight, ws, q_weight, k_weight, eps,
                                   interleaved, status, _stream(b.device(q if q is not None else k), stream)),
           "fpsk_qk_norm_rope_backward")


class QKNormRope(torch.autograd.Function):
    """qk_norm_rope with its gradients for autograd: ``apply(q, k, q_weight, k_weight, cos, sin, positions, out_dtype, eps,
    interleaved)`` returns the rotated queries and keys in out_dtype.  Gradients of q and k are computed and rounded once in
    their own type (in FP32 where it differs from out_dtype).  A second derivative is refused."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, out_dtype, eps, interleaved):
        q_out = torch.empty(q.shape, dtype=out_dtype, device=q.device)
        k_out = torch.empty(k.shape, dtype=out_dtype, device=k.device)
        qk_norm_rope(q, k, cos, sin, positions, q_out, k_out, q_weight, k_weight, eps, interleaved)
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.more = (out_dtype, eps, interleaved)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
        out_dtype, eps, interleaved = ctx.more
        # the library's gradients have one type: with an FP32 accumulator behind 16-bit outputs that is FP32, not the outputs'
        grad_dtype = out_dtype if q.dtype == out_dtype else torch.float32
        dq_out, dk_out = ((g if g.stride(-1) == 1 else g.contiguous()).to(grad_dtype) for g in (dq_out, dk_out))
        dq = torch.empty(q.shape, dtype=grad_dtype, device=q.device)
        dk = torch.empty(k.shape, dtype=grad_dtype, device=k.device)
        dw = [torch.empty(w.shape, dtype=torch.float32, device=w.device) if w is not None else None for w in (q_weight, k_weight)]
        qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dw[0], dw[1],
                              norm_rope_workspace(q.shape[2], q.device), q_weight, k_weight, eps, interleaved)
        dw = [g.to(w.dtype) if w is not None else None for g, w in zip(dw, (q_weight, k_weight))]
        return dq.to(q.dtype), dk.to(k.dtype), dw[0], dw[1], None, None, None, None, None, None


class PagedCache:
    """A cache of keys and values in pages: k and v are (pages, page size, key heads, dim) tensors of one 16-bit type, any
    strides with contiguous channels (a permuted view of (pages, key heads, page size, dim) works as well)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        self.device = (_binding or _bind()).check_cache(k, v)
        self.k, self.v = k, v


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                 block_table: torch.Tensor, cos=None, sin=None, k_weight=None, q=None, q_out=None, q_weight=None,
                 positions=None, eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """Writes the new tokens' keys (normed where k_weight is given, rotated) and values (tokens, key heads, dim) to their pages:
    token t of sequence b sits at position kv_len[b] - (cu_q[b + 1] - t); kv_len counts the new tokens.  With q, the queries
    are normed and rotated into q_out in the same launch.  Rotation goes by `positions` where given, else by that position."""
    _check(_binding.paged_append(cache.k, cache.v, k, v, cu_q, kv_len, block_table, cos, sin, k_weight, q, q_out, q_weight, positions, eps,
                                 interleaved, status, _stream(cache.device, stream)), "fpsk_paged_append")


def attention_workspace(device=None, stream=None) -> torch.Tensor:
    """Workspace of paged_attention, of one size for all calls on a device; serves one call at a time."""
    _bind()
    return _workspace(lambda: int(fpsk.lib().fpsk_paged_attention_workspace_bytes()), device, stream)


def paged_attention(cache: PagedCache, q: torch.Tensor, out: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                    block_table: torch.Tensor, ws: torch.Tensor, max_q_len: int, max_kv_len: int, scale: Optional[float] = None,
                    causal: bool = True, window: int = -1, lse: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of the new tokens q (tokens, query heads, dim) over their sequences' pages into `out` (and the log-sum-exp of
    their scores into lse, FP32 (tokens, query heads)).  A token at position p sees the keys j < kv_len with j <= p (causal)
    and j >= p - window (window >= 0); one that sees none gets zeros and -inf.  max_q_len and max_kv_len are upper bounds of
    the lengths, known to the host; they choose the tiling."""
    _check(_binding.paged_attention(cache.k, cache.v, q, out, cu_q, kv_len, block_table, ws, max_q_len, max_kv_len, scale, causal, window, lse,
                                    status, _stream(cache.device, stream)), "fpsk_paged_attention")
