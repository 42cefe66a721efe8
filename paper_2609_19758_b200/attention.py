"""The attention operators that follow a verified projection (``include/fpsk_attention.h``): norms and rotation of
queries and keys with their backward pass, writes to a paged cache, and attention of new tokens over it.

Argument marshalling only, like ``fpsk.py``: every step runs inside the CUDA library, asynchronously on the given (or
the current) stream.  Outputs and workspaces are the caller's tensors.
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional

import torch

from . import fpsk
from .fpsk import ERR_SHAPE, STATUS_OK, FpskError

ELEM = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}


class Rotary(C.Structure):
    _fields_ = [("cos", C.c_void_p), ("sin", C.c_void_p), ("positions", C.c_void_p), ("n_pos", C.c_int64),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32)]


class Heads(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("weight", C.c_void_p), ("in_token_stride", C.c_int64),
                ("in_head_stride", C.c_int64), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64),
                ("n_heads", C.c_int32), ("weight_type", C.c_int32)]


class HeadsGrad(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("dout", C.c_void_p), ("din", C.c_void_p), ("weight", C.c_void_p), ("dweight", C.c_void_p),
                ("in_token_stride", C.c_int64), ("in_head_stride", C.c_int64), ("dout_token_stride", C.c_int64),
                ("dout_head_stride", C.c_int64), ("din_token_stride", C.c_int64), ("din_head_stride", C.c_int64),
                ("n_heads", C.c_int32), ("weight_type", C.c_int32)]


class Cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_page_stride", C.c_int64), ("k_token_stride", C.c_int64),
                ("k_head_stride", C.c_int64), ("v_page_stride", C.c_int64), ("v_token_stride", C.c_int64),
                ("v_head_stride", C.c_int64), ("n_pages", C.c_int64), ("page_size", C.c_int32), ("n_heads", C.c_int32),
                ("head_dim", C.c_int32), ("type", C.c_int32)]


class Batch(C.Structure):
    _fields_ = [("cu_q", C.c_void_p), ("kv_len", C.c_void_p), ("block_table", C.c_void_p), ("table_stride", C.c_int64),
                ("n_tokens", C.c_int64), ("n_seqs", C.c_int32), ("max_pages", C.c_int32)]


class Attention(C.Structure):
    _fields_ = [("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("q_token_stride", C.c_int64),
                ("q_head_stride", C.c_int64), ("out_token_stride", C.c_int64), ("out_head_stride", C.c_int64),
                ("n_heads", C.c_int32), ("causal", C.c_int32), ("window", C.c_int32), ("max_q_len", C.c_int32),
                ("max_kv_len", C.c_int32), ("scale", C.c_float)]


_bound = None


def _lib() -> C.CDLL:
    global _bound
    if _bound is None:
        L = fpsk.lib()
        vp, i64, i32, sz, P = C.c_void_p, C.c_int64, C.c_int32, C.c_size_t, C.POINTER
        for name, restype, argtypes in (
                ("fpsk_qk_norm_rope", C.c_int, [P(Heads), P(Heads), i64, i32, C.c_int, C.c_int, P(Rotary), C.c_float, vp, vp]),
                ("fpsk_norm_rope_workspace_bytes", sz, [i32]),
                ("fpsk_qk_norm_rope_backward", C.c_int, [P(HeadsGrad), P(HeadsGrad), i64, i32, C.c_int, C.c_int, P(Rotary),
                                                         C.c_float, vp, sz, vp, vp]),
                ("fpsk_paged_append", C.c_int, [P(Cache), P(Batch), P(Heads), P(Heads), P(Heads), C.c_int, P(Rotary), C.c_float,
                                                vp, vp]),
                ("fpsk_paged_attention_workspace_bytes", sz, []),
                ("fpsk_paged_attention", C.c_int, [P(Cache), P(Batch), P(Attention), vp, sz, vp, vp]),
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


def _stream(t: torch.Tensor, stream) -> int:
    """The given stream, else the current one of the tensor's device."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(t.device.index)


def _elem(t: torch.Tensor) -> int:
    e = ELEM.get(t.dtype)
    if e is None:
        raise TypeError(f"float16, bfloat16 or float32 expected, got {t.dtype}")
    return e


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _same(t: Optional[torch.Tensor], shape, dtype, what: str, device) -> None:
    """t has this shape (None entries: any), type and device, its channels contiguous."""
    if t is None:
        return
    if tuple(t.shape) != shape or t.dtype != dtype or t.device != device or (t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what}: expected {shape} {dtype} on {device} with contiguous channels, "
                         f"got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")


def _index(t: torch.Tensor, dims: int, what: str, device) -> None:
    if t.dtype != torch.int32 or t.dim() != dims or t.device != device or (t.stride(-1) != 1 and t.shape[-1] > 1):
        raise ValueError(f"{what}: expected a {dims}-dimensional contiguous int32 tensor on {device}")


def _rotary(cos, sin, positions, interleaved, n_tokens, device) -> Rotary:
    r = Rotary()
    if cos is None or cos.shape[1] == 0:
        return r
    _need(sin is not None and cos.shape == sin.shape and cos.dtype == sin.dtype == torch.float32 and cos.is_contiguous()
          and sin.is_contiguous() and cos.device == sin.device == device, "cos, sin: contiguous FP32 tables (positions, rot_dim / 2)")
    if positions is not None:
        _index(positions, 1, "positions", device)
        _need(positions.shape[0] == n_tokens, "positions: one per token")
        r.positions = positions.data_ptr()
    r.cos, r.sin, r.n_pos, r.rot_dim, r.interleaved = cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1], int(interleaved)
    return r


def _heads(x: Optional[torch.Tensor], out: Optional[torch.Tensor], weight: Optional[torch.Tensor], like: torch.Tensor,
           out_dtype, what: str) -> Heads:
    h = Heads()
    if x is None:
        return h
    n, heads, dim = x.shape
    _same(x, (like.shape[0], heads, like.shape[2]), like.dtype, what, like.device)
    s = x.stride()
    h.in_, h.in_token_stride, h.in_head_stride, h.n_heads = x.data_ptr(), s[0], s[1], heads
    if out is not None:
        _same(out, (n, heads, dim), out_dtype, what + "_out", like.device)
        s = out.stride()
        h.out, h.out_token_stride, h.out_head_stride = out.data_ptr(), s[0], s[1]
    if weight is not None:
        _need(tuple(weight.shape) == (dim,) and weight.is_contiguous() and weight.device == like.device, f"{what}_weight: ({dim},)")
        h.weight, h.weight_type = weight.data_ptr(), _elem(weight)
    return h


def _workspace(nbytes: int, device, stream) -> torch.Tensor:
    ws = torch.empty(nbytes, dtype=torch.uint8, device=device or "cuda")
    _check(_lib().fpsk_attention_workspace_init(ws.data_ptr(), nbytes, _stream(ws, stream)), "fpsk_attention_workspace_init")
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
    like = q if q is not None else k
    out = q_out if q is not None else k_out
    hq = _heads(q, q_out, q_weight, like, out.dtype, "q")
    hk = _heads(k, k_out, k_weight, like, out.dtype, "k")
    r = _rotary(cos, sin, positions, interleaved, like.shape[0], like.device)
    _check(_lib().fpsk_qk_norm_rope(hq, hk, like.shape[0], like.shape[2], _elem(like), _elem(out), r, eps, _ptr(status),
                                    _stream(like, stream)), "fpsk_qk_norm_rope")


def norm_rope_workspace(head_dim: int, device=None, stream=None) -> torch.Tensor:
    """Workspace of qk_norm_rope_backward; serves one call at a time."""
    n = int(_lib().fpsk_norm_rope_workspace_bytes(head_dim))
    if n == 0:
        raise FpskError(ERR_SHAPE, "fpsk_norm_rope_workspace_bytes")
    return _workspace(n, device, stream)


def _heads_grad(x, dy, dx, weight, dweight, like, grad_dtype, what: str) -> HeadsGrad:
    h = HeadsGrad()
    if x is None:
        return h
    n, heads, dim = x.shape
    _same(x, (like.shape[0], heads, like.shape[2]), like.dtype, what, like.device)
    _same(dy, (n, heads, dim), grad_dtype, f"d{what}_out", like.device)
    _same(dx, (n, heads, dim), grad_dtype, f"d{what}", like.device)
    s, t, u = x.stride(), dy.stride(), dx.stride()
    h.in_, h.in_token_stride, h.in_head_stride, h.n_heads = x.data_ptr(), s[0], s[1], heads
    h.dout, h.dout_token_stride, h.dout_head_stride = dy.data_ptr(), t[0], t[1]
    h.din, h.din_token_stride, h.din_head_stride = dx.data_ptr(), u[0], u[1]
    if weight is not None:
        _need(tuple(weight.shape) == (dim,) and weight.is_contiguous() and weight.device == like.device, f"{what}_weight: ({dim},)")
        _need(dweight is not None and tuple(dweight.shape) == (dim,) and dweight.dtype == torch.float32 and dweight.is_contiguous()
              and dweight.device == like.device, f"d{what}_weight: FP32 ({dim},)")
        h.weight, h.weight_type, h.dweight = weight.data_ptr(), _elem(weight), dweight.data_ptr()
    return h


def qk_norm_rope_backward(q, k, dq_out, dk_out, cos, sin, positions, dq, dk, dq_weight, dk_weight, ws: torch.Tensor,
                          q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                          status: Optional[torch.Tensor] = None, stream=None) -> None:
    """Backward pass of qk_norm_rope from its inputs q, k and the gradients of its outputs: fills dq, dk (the type of dq_out)
    and the FP32 gradients of the weights (overwritten)."""
    like = q if q is not None else k
    g = dq_out if q is not None else dk_out
    hq = _heads_grad(q, dq_out, dq, q_weight, dq_weight, like, g.dtype, "q")
    hk = _heads_grad(k, dk_out, dk, k_weight, dk_weight, like, g.dtype, "k")
    r = _rotary(cos, sin, positions, interleaved, like.shape[0], like.device)
    _check(_lib().fpsk_qk_norm_rope_backward(hq, hk, like.shape[0], like.shape[2], _elem(like), _elem(g), r, eps, ws.data_ptr(),
                                             ws.numel(), _ptr(status), _stream(like, stream)), "fpsk_qk_norm_rope_backward")


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
        c = self.c = Cache()
        c.k, c.v = k.data_ptr(), v.data_ptr()
        c.k_page_stride, c.k_token_stride, c.k_head_stride = k.stride()[:3]
        c.v_page_stride, c.v_token_stride, c.v_head_stride = v.stride()[:3]
        c.n_pages, c.page_size, c.n_heads, c.head_dim = k.shape
        c.type = ELEM[k.dtype]


def _batch(cu_q, kv_len, block_table, n_tokens, device) -> Batch:
    _index(cu_q, 1, "cu_q", device)
    _index(kv_len, 1, "kv_len", device)
    _index(block_table, 2, "block_table", device)
    n = kv_len.shape[0]
    _need(cu_q.shape[0] == n + 1 and block_table.shape[0] == n, "cu_q: (sequences + 1,), block_table: (sequences, pages)")
    b = Batch()
    b.cu_q, b.kv_len, b.block_table = cu_q.data_ptr(), kv_len.data_ptr(), block_table.data_ptr()
    b.max_pages = block_table.shape[1]
    b.table_stride = max(block_table.stride(0), b.max_pages) if n > 1 else b.max_pages
    b.n_tokens, b.n_seqs = n_tokens, n
    return b


def paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, cu_q: torch.Tensor, kv_len: torch.Tensor,
                 block_table: torch.Tensor, cos=None, sin=None, k_weight=None, q=None, q_out=None, q_weight=None,
                 positions=None, eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """Writes the new tokens' keys (normed where k_weight is given, rotated) and values (tokens, key heads, dim) to their pages:
    token t of sequence b sits at position kv_len[b] - (cu_q[b + 1] - t); kv_len counts the new tokens.  With q, the queries
    are normed and rotated into q_out in the same launch.  Rotation goes by `positions` where given, else by that position."""
    _same(k, (k.shape[0], cache.c.n_heads, cache.c.head_dim), k.dtype, "k", cache.k.device)
    _same(v, tuple(k.shape), k.dtype, "v", cache.k.device)
    hk = _heads(k, None, k_weight, k, None, "k")
    hv = _heads(v, None, None, k, None, "v")
    hq = _heads(q, q_out, q_weight, k, cache.k.dtype, "q")
    r = _rotary(cos, sin, positions, interleaved, k.shape[0], k.device)
    b = _batch(cu_q, kv_len, block_table, k.shape[0], k.device)
    _check(_lib().fpsk_paged_append(cache.c, b, hk, hv, hq, _elem(k), r, eps, _ptr(status), _stream(k, stream)), "fpsk_paged_append")


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
    n, heads, dim = q.shape
    _same(q, (n, heads, cache.c.head_dim), cache.k.dtype, "q", cache.k.device)
    _same(out, (n, heads, dim), cache.k.dtype, "out", q.device)
    a = Attention()
    if lse is not None:
        _same(lse, (n, heads), torch.float32, "lse", q.device)
        _need(lse.is_contiguous(), "lse must be contiguous")
        a.lse = lse.data_ptr()
    s, t = q.stride(), out.stride()
    a.q, a.q_token_stride, a.q_head_stride = q.data_ptr(), s[0], s[1]
    a.out, a.out_token_stride, a.out_head_stride = out.data_ptr(), t[0], t[1]
    a.n_heads, a.causal, a.window, a.max_q_len, a.max_kv_len = heads, int(causal), window, max_q_len, max_kv_len
    if scale is not None:
        _need(scale > 0 and math.isfinite(scale), "scale must be positive and finite")
        a.scale = scale
    b = _batch(cu_q, kv_len, block_table, n, q.device)
    _check(_lib().fpsk_paged_attention(cache.c, b, a, ws.data_ptr(), ws.numel(), _ptr(status), _stream(q, stream)), "fpsk_paged_attention")
