"""The attention operators that follow a verified projection (``include/fpsk_attention.h``): norms and rotation of
queries and keys with their backward pass, writes to a paged cache, and attention of new tokens over it.

Argument marshalling only, like ``fpsk.py``: every step runs inside the CUDA library, asynchronously on the given (or
the current) stream.  Outputs and workspaces are the caller's tensors.
"""
from __future__ import annotations

import ctypes as C
import math
from struct import Struct
from typing import Optional

import torch

from . import fpsk
from .fpsk import ERR_SHAPE, STATUS_OK, FpskError

ELEM = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


# The structs of the header as packed bytes (a call's arguments are built in a microsecond or two this way; ctypes takes bytes
# where the library takes a pointer).
_HEADS = Struct("@PPPqqqqii")                # fpsk_heads
_HEADS_GRAD = Struct("@PPPPPqqqqqqii")       # fpsk_heads_grad
_ROTARY = Struct("@PPPqii")                  # fpsk_rotary
_CACHE = Struct("@PPqqqqqqqiiii")            # fpsk_paged_cache
_BATCH = Struct("@PPPqqii")                  # fpsk_paged_batch
_ATTENTION = Struct("@PPPqqqqiiiiif")        # fpsk_attention
_NO_ROTARY = bytes(_ROTARY.size)

_bound = None


def _lib() -> C.CDLL:
    global _bound
    if _bound is None:
        L = fpsk.lib()
        vp, i64, i32, sz = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t
        for name, restype, argtypes in (
                ("fpsk_qk_norm_rope", C.c_int, [vp, vp, i64, i32, C.c_int, C.c_int, vp, C.c_float, vp, vp]),
                ("fpsk_norm_rope_workspace_bytes", sz, [i32]),
                ("fpsk_qk_norm_rope_backward", C.c_int, [vp, vp, i64, i32, C.c_int, C.c_int, vp, C.c_float, vp, sz, vp, vp]),
                ("fpsk_paged_append", C.c_int, [vp, vp, vp, vp, vp, C.c_int, vp, C.c_float, vp, vp]),
                ("fpsk_paged_attention_workspace_bytes", sz, []),
                ("fpsk_paged_attention", C.c_int, [vp, vp, vp, vp, sz, vp, vp]),
                ("fpsk_attention_workspace_init", C.c_int, [vp, sz, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = restype, argtypes
        _bound = L
    return _bound


def _check(rc: int, where: str) -> None:
    if rc != STATUS_OK:
        raise FpskError(rc, where)


def _ptr(t: Optional[torch.Tensor]):
    return t.data_ptr() if t is not None else None


def _stream(device: int, stream) -> int:
    """The given stream, else the current one of the device."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(device)


def _elem(dtype) -> int:
    e = ELEM.get(dtype)
    if e is None:
        raise TypeError(f"float16, bfloat16 or float32 expected, got {dtype}")
    return e


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _strides(t: torch.Tensor, shape, dtype, device: int, what: str):
    """The strides of t, which has this shape, type and device and contiguous channels."""
    s = t.stride()
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or (s[-1] != 1 and shape[-1] > 1):
        raise ValueError(f"{what}: expected {tuple(shape)} {dtype} on cuda:{device} with contiguous channels, "
                         f"got {tuple(t.shape)} {t.dtype} on {t.device}, strides {s}")
    return s


def _index(t: torch.Tensor, dims: int, device: int, what: str):
    """The shape of an int32 index tensor with a contiguous last dimension."""
    n = t.shape
    if t.dtype is not torch.int32 or len(n) != dims or t.get_device() != device or (n[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what}: expected a {dims}-dimensional contiguous int32 tensor on cuda:{device}")
    return n


def _rotary(cos, sin, positions, interleaved, n_tokens: int, device: int) -> bytes:
    if cos is None:
        return _NO_ROTARY
    n_pos, half = cos.shape
    if half == 0:
        return _NO_ROTARY
    if (sin is None or sin.shape != cos.shape or cos.dtype is not torch.float32 or sin.dtype is not torch.float32
            or not cos.is_contiguous() or not sin.is_contiguous() or cos.get_device() != device or sin.get_device() != device):
        raise ValueError("cos, sin: contiguous FP32 tables (positions, rot_dim / 2)")
    at = 0
    if positions is not None:
        _need(_index(positions, 1, device, "positions")[0] == n_tokens, "positions: one per token")
        at = positions.data_ptr()
    return _ROTARY.pack(cos.data_ptr(), sin.data_ptr(), at, n_pos, 2 * half, 1 if interleaved else 0)


def _weight(w: Optional[torch.Tensor], dim: int, device: int, what: str):
    if w is None:
        return 0, 0
    if w.shape != (dim,) or w.get_device() != device or not w.is_contiguous():
        raise ValueError(f"{what}_weight: contiguous ({dim},) on cuda:{device}")
    return w.data_ptr(), _elem(w.dtype)


def _heads(x: Optional[torch.Tensor], out: Optional[torch.Tensor], weight: Optional[torch.Tensor], like: torch.Tensor,
           out_dtype, device: int, what: str):
    if x is None:
        return None
    n, heads, dim = shape = x.shape
    full = like.shape
    if x is not like and (n != full[0] or dim != full[2]):
        raise ValueError(f"{what}: expected {full[0]} tokens and heads of {full[2]}, got {tuple(shape)}")
    s = _strides(x, shape, like.dtype, device, what)
    to, t = 0, s
    if out is not None:
        t = _strides(out, shape, out_dtype, device, what + "_out")
        to = out.data_ptr()
    w, w_type = _weight(weight, dim, device, what)
    return _HEADS.pack(x.data_ptr(), to, w, s[0], s[1], t[0], t[1], heads, w_type)


def _workspace(nbytes: int, device, stream) -> torch.Tensor:
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")
    _check(_lib().fpsk_attention_workspace_init(ws.data_ptr(), nbytes, _stream(ws.get_device(), stream)), "fpsk_attention_workspace_init")
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
    like, out = (q, q_out) if q is not None else (k, k_out)
    device, out_dtype = like.get_device(), out.dtype
    n, _, dim = like.shape
    hq = _heads(q, q_out, q_weight, like, out_dtype, device, "q")
    hk = _heads(k, k_out, k_weight, like, out_dtype, device, "k")
    r = _rotary(cos, sin, positions, interleaved, n, device)
    _check(_lib().fpsk_qk_norm_rope(hq, hk, n, dim, _elem(like.dtype), _elem(out_dtype), r, eps, _ptr(status),
                                    _stream(device, stream)), "fpsk_qk_norm_rope")


def norm_rope_workspace(head_dim: int, device=None, stream=None) -> torch.Tensor:
    """Workspace of qk_norm_rope_backward; serves one call at a time."""
    n = int(_lib().fpsk_norm_rope_workspace_bytes(head_dim))
    if n == 0:
        raise FpskError(ERR_SHAPE, "fpsk_norm_rope_workspace_bytes")
    return _workspace(n, device, stream)


def _heads_grad(x, dy, dx, weight, dweight, like, grad_dtype, device: int, what: str):
    if x is None:
        return None
    n, heads, dim = shape = x.shape
    full = like.shape
    if x is not like and (n != full[0] or dim != full[2]):
        raise ValueError(f"{what}: expected {full[0]} tokens and heads of {full[2]}, got {tuple(shape)}")
    s = _strides(x, shape, like.dtype, device, what)
    t = _strides(dy, shape, grad_dtype, device, f"d{what}_out")
    u = _strides(dx, shape, grad_dtype, device, f"d{what}")
    w, w_type = _weight(weight, dim, device, what)
    dw = 0
    if w:
        _need(dweight is not None and dweight.shape == (dim,) and dweight.dtype is torch.float32 and dweight.is_contiguous()
              and dweight.get_device() == device, f"d{what}_weight: FP32 ({dim},)")
        dw = dweight.data_ptr()
    return _HEADS_GRAD.pack(x.data_ptr(), dy.data_ptr(), dx.data_ptr(), w, dw, s[0], s[1], t[0], t[1], u[0], u[1], heads, w_type)


def qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dq_weight, dk_weight, ws: torch.Tensor,
                          q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                          status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward pass of qk_norm_rope from its inputs q, k and the gradients of its outputs: fills dq, dk (the type of dq_out)
    and the FP32 gradients of the weights (overwritten)."""
    like, g = (q, dq_out) if q is not None else (k, dk_out)
    device, grad_dtype = like.get_device(), g.dtype
    n, _, dim = like.shape
    hq = _heads_grad(q, dq_out, dq, q_weight, dq_weight, like, grad_dtype, device, "q")
    hk = _heads_grad(k, dk_out, dk, k_weight, dk_weight, like, grad_dtype, device, "k")
    r = _rotary(cos, sin, positions, interleaved, n, device)
    _check(_lib().fpsk_qk_norm_rope_backward(hq, hk, n, dim, _elem(like.dtype), _elem(grad_dtype), r, eps, ws.data_ptr(),
                                             ws.numel(), _ptr(status), _stream(device, stream)), "fpsk_qk_norm_rope_backward")


class QKNormRope(torch.autograd.Function):
    """qk_norm_rope with its gradients for autograd: ``apply(q, k, q_weight, k_weight, cos, sin, positions, out_dtype, eps,
    interleaved)`` returns the rotated queries and keys in out_dtype.  Gradients of q and k are computed in out_dtype."""

    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, cos, sin, positions, out_dtype, eps, interleaved):
        q_out = torch.empty(q.shape, dtype=out_dtype, device=q.device)
        k_out = torch.empty(k.shape, dtype=out_dtype, device=k.device)
        qk_norm_rope(q, k, cos, sin, positions, q_out, k_out, q_weight, k_weight, eps, interleaved)
        ctx.save_for_backward(q, k, q_weight, k_weight, cos, sin, positions)
        ctx.more = (out_dtype, eps, interleaved)
        return q_out, k_out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
        out_dtype, eps, interleaved = ctx.more
        dq_out, dk_out = (g if g.stride(-1) == 1 else g.contiguous() for g in (dq_out, dk_out))
        dq = torch.empty(q.shape, dtype=out_dtype, device=q.device)
        dk = torch.empty(k.shape, dtype=out_dtype, device=k.device)
        dw = [torch.empty(w.shape, dtype=torch.float32, device=w.device) if w is not None else None for w in (q_weight, k_weight)]
        qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dw[0], dw[1],
                              norm_rope_workspace(q.shape[2], q.device), q_weight, k_weight, eps, interleaved)
        dw = [g.to(w.dtype) if w is not None else None for g, w in zip(dw, (q_weight, k_weight))]
        return dq.to(q.dtype), dk.to(k.dtype), dw[0], dw[1], None, None, None, None, None, None


class PagedCache:
    """A cache of keys and values in pages: k and v are (pages, page size, key heads, dim) tensors of one 16-bit type, any
    strides with contiguous channels (a permuted view of (pages, key heads, page size, dim) works as well)."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        _need(k.dim() == 4 and k.is_cuda and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device, "k, v: two alike tensors (pages, page size, heads, dim)")
        _need(k.dtype in (torch.float16, torch.bfloat16), "a cache is float16 or bfloat16")
        _need(k.stride(3) == 1 and v.stride(3) == 1, "channels must be contiguous")
        self.k, self.v = k, v
        self.n_heads, self.head_dim, self.dtype, self.device = k.shape[2], k.shape[3], k.dtype, k.get_device()
        self.packed = _CACHE.pack(k.data_ptr(), v.data_ptr(), *k.stride()[:3], *v.stride()[:3], *k.shape, ELEM[k.dtype])


def _batch(cu_q, kv_len, block_table, n_tokens: int, device: int) -> bytes:
    n, = _index(kv_len, 1, device, "kv_len")
    rows, pages = _index(block_table, 2, device, "block_table")
    _need(_index(cu_q, 1, device, "cu_q")[0] == n + 1 and rows == n, "cu_q: (sequences + 1,), block_table: (sequences, pages)")
    return _BATCH.pack(cu_q.data_ptr(), kv_len.data_ptr(), block_table.data_ptr(), max(block_table.stride(0), pages) if n > 1 else pages,
                       n_tokens, n, pages)


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                 block_table: torch.Tensor, cos=None, sin=None, k_weight=None, q=None, q_out=None, q_weight=None,
                 positions=None, eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """Writes the new tokens' keys (normed where k_weight is given, rotated) and values (tokens, key heads, dim) to their pages:
    token t of sequence b sits at position kv_len[b] - (cu_q[b + 1] - t); kv_len counts the new tokens.  With q, the queries
    are normed and rotated into q_out in the same launch.  Rotation goes by `positions` where given, else by that position."""
    device, n = cache.device, k.shape[0]
    _need(k.shape[1:] == (cache.n_heads, cache.head_dim) and v.shape == k.shape,
          f"k, v: expected (tokens, {cache.n_heads}, {cache.head_dim}), got {tuple(k.shape)}, {tuple(v.shape)}")
    hk = _heads(k, None, k_weight, k, None, device, "k")
    hv = _heads(v, None, None, k, None, device, "v")
    hq = _heads(q, q_out, q_weight, k, cache.dtype, device, "q")
    r = _rotary(cos, sin, positions, interleaved, n, device)
    b = _batch(cu_q, kv_len, block_table, n, device)
    _check(_lib().fpsk_paged_append(cache.packed, b, hk, hv, hq, _elem(k.dtype), r, eps, _ptr(status), _stream(device, stream)),
           "fpsk_paged_append")


def attention_workspace(device=None, stream=None) -> torch.Tensor:
    """Workspace of paged_attention, of one size for all calls on a device; serves one call at a time."""
    return _workspace(int(_lib().fpsk_paged_attention_workspace_bytes()), device, stream)


def paged_attention(cache: PagedCache, q: torch.Tensor, out: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                    block_table: torch.Tensor, ws: torch.Tensor, max_q_len: int, max_kv_len: int, scale: Optional[float] = None,
                    causal: bool = True, window: int = -1, lse: Optional[torch.Tensor] = None,
                    status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Attention of the new tokens q (tokens, query heads, dim) over their sequences' pages into `out` (and the log-sum-exp of
    their scores into lse, FP32 (tokens, query heads)).  A token at position p sees the keys j < kv_len with j <= p (causal)
    and j >= p - window (window >= 0); one that sees none gets zeros and -inf.  max_q_len and max_kv_len are upper bounds of
    the lengths, known to the host; they choose the tiling."""
    n, heads, dim = shape = q.shape
    device = cache.device
    _need(dim == cache.head_dim, f"q: expected heads of {cache.head_dim}, got {dim}")
    s = _strides(q, shape, cache.dtype, device, "q")
    t = _strides(out, shape, cache.dtype, device, "out")
    to = 0
    if lse is not None:
        _strides(lse, (n, heads), torch.float32, device, "lse")
        _need(lse.is_contiguous(), "lse must be contiguous")
        to = lse.data_ptr()
    if scale is None:
        scale = 0.0
    else:
        _need(scale > 0 and math.isfinite(scale), "scale must be positive and finite")
    a = _ATTENTION.pack(q.data_ptr(), out.data_ptr(), to, s[0], s[1], t[0], t[1], heads, 1 if causal else 0, window, max_q_len, max_kv_len,
                        scale)
    b = _batch(cu_q, kv_len, block_table, n, device)
    _check(_lib().fpsk_paged_attention(cache.packed, b, a, ws.data_ptr(), ws.numel(), _ptr(status), _stream(device, stream)),
           "fpsk_paged_attention")
