"""Host-side checks of the decoder operators' C ABI that need no GPU: struct layouts and argument validation."""
import ctypes as C
import struct

import pytest

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

F16, BF16, F32, E4M3 = 0, 1, 2, 3
vp, sz = C.c_void_p, C.c_size_t
P = 4096                                                               # never read: validation fails first


@pytest.fixture(scope="module")
def lib():
    B.build()
    L = fpsk.lib()
    L.fpsk_add_rms_norm.argtypes = [vp, vp, vp]
    L.fpsk_add_rms_norm_backward.argtypes = [vp, vp, sz, vp, vp]
    L.fpsk_add_norm_workspace_bytes.argtypes, L.fpsk_add_norm_workspace_bytes.restype = [C.c_int32], sz
    L.fpsk_adjust_logits.argtypes = [vp, vp, vp]
    L.fpsk_distill_loss.argtypes = L.fpsk_distill_loss_backward.argtypes = [vp, vp, vp]
    return L


def test_add_norm(lib):
    def call(x=P, res=0, w=0, hout=0, y=P, scale=0, strides=(64, 64, 64, 64, 1), n=2, dim=64, types=(F32, F32, F32, F32), group=0, eps=1e-6):
        return lib.fpsk_add_rms_norm(struct.pack("@PPPPPPqqqqqqiiiiiif", x, res, w, hout, y, scale, *strides, n, dim, *types, group, eps), None, None)

    assert lib.fpsk_add_rms_norm(None, None, None) == fpsk.ERR_NULL
    assert call(n=-1) == call(dim=0) == call(dim=32769) == call(strides=(64, 64, 64, 63, 1)) == call(strides=(-1, 64, 64, 64, 1)) == fpsk.ERR_SHAPE
    assert call(hout=P, strides=(64, 64, 60, 64, 1)) == fpsk.ERR_SHAPE
    assert call(types=(E4M3, 0, 0, 0)) == call(res=P, types=(F32, 3, 0, 0)) == call(w=P, types=(F32, 0, 4, 0)) == call(types=(F32, 0, 0, 4)) == fpsk.ERR_DTYPE
    assert call(eps=-1.0) == call(eps=float("nan")) == call(eps=float("inf")) == call(group=64) == fpsk.ERR_PARAM
    assert call(types=(F32, 0, 0, E4M3), group=48, scale=P) == call(types=(F32, 0, 0, E4M3), group=-32, scale=P) == fpsk.ERR_PARAM
    assert call(x=0) == call(y=0) == call(types=(F32, 0, 0, E4M3)) == fpsk.ERR_NULL
    assert call(types=(F32, 0, 0, E4M3), group=32, scale=P, strides=(64, 64, 64, 64, 1)) == fpsk.ERR_SHAPE
    assert call(x=P + 2) == call(res=P + 1) == call(w=P + 1) == call(y=P + 2) == fpsk.ERR_ALIGN
    assert call(n=0, x=0, y=0) == fpsk.STATUS_OK


def test_add_norm_backward(lib):
    def call(h=P, dy=P, dh=0, w=0, dx=P, dw=0, strides=(64, 64, 64, 64), n=2, dim=64, types=(F32, F32, F32), eps=1e-6, ws=0, ws_bytes=0):
        return lib.fpsk_add_rms_norm_backward(struct.pack("@PPPPPPqqqqqiiiif", h, dy, dh, w, dx, dw, *strides, n, dim, *types, eps), ws, ws_bytes, None, None)

    assert lib.fpsk_add_rms_norm_backward(None, None, 0, None, None) == fpsk.ERR_NULL
    assert lib.fpsk_add_norm_workspace_bytes(0) == lib.fpsk_add_norm_workspace_bytes(32769) == 0 < lib.fpsk_add_norm_workspace_bytes(64)
    assert call(n=-1) == call(dim=0) == call(strides=(64, 64, 64, 8)) == call(strides=(64, -64, 64, 64)) == fpsk.ERR_SHAPE
    assert call(types=(E4M3, 0, 0)) == call(types=(F32, E4M3, 0)) == call(w=P, types=(F32, F32, 7)) == fpsk.ERR_DTYPE
    assert call(eps=-1e-9) == fpsk.ERR_PARAM
    assert call(h=0) == call(dy=0) == call(dx=0) == call(dw=P) == fpsk.ERR_NULL
    assert call(dw=P, ws=P + 16, ws_bytes=1 << 30) == fpsk.ERR_ALIGN
    assert call(dw=P, ws=P, ws_bytes=255) == fpsk.ERR_WORKSPACE
    assert call(h=P + 2) == call(dy=P + 1) == call(dh=P + 2) == call(dx=P + 3) == fpsk.ERR_ALIGN
    assert call(n=0, h=0, dy=0, dx=0) == fpsk.STATUS_OK


def test_adjust_logits(lib):
    def call(x=P, out=P, strides=(100, 100), n=2, vocab=100, types=(F32, F32), width=0, history=(0, 0, 0), history_stride=0, penalties=(0, 0, 0),
             bias=(0, 0, 0), n_biases=0, mask=(0, 0), mask_stride=4, n_masks=2, token=0, lse=0):
        s = struct.pack("@PPqqqiiiiPPPqPPPPPPqPPqqPP", x, out, *strides, n, vocab, *types, width, *history, history_stride, *penalties, *bias, n_biases, *mask,
                        mask_stride, n_masks, token, lse)
        return lib.fpsk_adjust_logits(s, None, None)

    assert lib.fpsk_adjust_logits(None, None, None) == fpsk.ERR_NULL
    assert call(n=-1) == call(n=1 << 31) == call(vocab=0) == call(vocab=(1 << 23) + 1) == call(strides=(100, 99)) == call(strides=(-1, 100)) == fpsk.ERR_SHAPE
    assert call(types=(E4M3, F32)) == call(types=(F32, E4M3)) == fpsk.ERR_DTYPE
    assert call(x=0) == call(out=0) == call(penalties=(P, 0, 0)) == call(history=(0, P, 0)) == call(bias=(P, 0, P), n_biases=3) == call(mask=(0, P)) == fpsk.ERR_NULL
    assert call(x=P + 2) == call(out=P + 1) == fpsk.ERR_ALIGN
    assert call(history=(P, 0, 0), width=-1) == call(history=(P, 0, 0), width=(1 << 28) + 1) == call(mask=(P, 0), mask_stride=-1) == fpsk.ERR_SHAPE
    assert call(mask=(P, 0), mask_stride=4, n_masks=1) == fpsk.ERR_SHAPE            # fewer masks than rows, and nothing says whose
    assert call(n=0, x=0) == fpsk.STATUS_OK


def test_distill(lib):
    def call(f, x=P, tok=P, t=P, weight=0, loss=P, lse=P, dx=P, strides=(100, 4, 4, 100), n=2, vocab=100, top=4, types=(F32, 4, F32, F32), normalize=1, tau=1.0):
        return f(struct.pack("@PPPPPPPqqqqqiiiiiiif", x, tok, t, weight, loss, lse, dx, *strides, n, vocab, top, *types, normalize, tau), None, None)

    for f in (lib.fpsk_distill_loss, lib.fpsk_distill_loss_backward):
        assert f(None, None, None) == fpsk.ERR_NULL
        assert call(f, n=-1) == call(f, vocab=0) == call(f, top=-1) == call(f, top=1025) == call(f, strides=(100, 4, 4, 99)) == call(f, strides=(-1, 4, 4, 100)) == fpsk.ERR_SHAPE
        assert call(f, types=(E4M3, 4, F32, F32)) == call(f, types=(F32, 2, F32, F32)) == call(f, types=(F32, 8, E4M3, F32)) == call(f, types=(F32, 8, F32, E4M3)) == fpsk.ERR_DTYPE
        assert call(f, tau=0.0) == call(f, tau=-1.0) == call(f, tau=float("nan")) == call(f, tau=float("inf")) == call(f, tau=1e-39) == fpsk.ERR_PARAM
        assert call(f, x=P + 2) == call(f, dx=P + 2) == fpsk.ERR_ALIGN
        assert call(f, x=0) == call(f, tok=0) == call(f, t=0) == fpsk.ERR_NULL
        assert call(f, n=0, x=0) == fpsk.STATUS_OK
    assert call(lib.fpsk_distill_loss, loss=0) == call(lib.fpsk_distill_loss_backward, lse=0) == call(lib.fpsk_distill_loss_backward, dx=0) == fpsk.ERR_NULL


def test_binding_refuses_tensors_of_the_host():
    import torch
    from paper_2609_19758_b200 import logits as L
    from paper_2609_19758_b200 import norm as N
    x = torch.zeros(2, 16)
    for bad in (lambda: N.add_rms_norm(x, None, None, x.clone()), lambda: N.add_rms_norm_backward(x, x, None, x.clone()), lambda: L.adjust_logits(x, x),
                lambda: L.distill_loss(x, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1), torch.zeros(2))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(TypeError):
        N.add_rms_norm("x", None, None, x)
