"""Host-side checks of the decoder operators' C ABI: pointers that their types may not have are refused before a launch, temperatures whose
powers FP32 does not hold as well."""
import ctypes as C
import struct

import pytest

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

F16, BF16, F32 = 0, 1, 2
P = 4096                                                               # never read: validation fails first


@pytest.fixture(scope="module")
def lib():
    B.build()
    L = fpsk.lib()
    for f in (L.fpsk_adjust_logits, L.fpsk_distill_loss, L.fpsk_distill_loss_backward):
        f.argtypes = [C.c_void_p] * 3
    return L


FIELDS = ["history", "history_len", "prompt_len", "repetition", "frequency", "presence", "bias_ptr", "bias_token", "bias_value", "mask", "mask_row", "token", "lse"]


@pytest.mark.parametrize("field", FIELDS)
@pytest.mark.parametrize("off", [1, 2])
def test_logits(lib, field, off):
    p = {n: P + off * (n == field) for n in FIELDS}
    s = struct.pack("@PPqqqiiiiPPPqPPPPPPqPPqqPP", P, P, 100, 100, 2, 100, F32, F32, 5, p["history"], p["history_len"], p["prompt_len"], 5, p["repetition"],
                    p["frequency"], p["presence"], p["bias_ptr"], p["bias_token"], p["bias_value"], 3, p["mask"], p["mask_row"], 4, 2, p["token"], p["lse"])
    assert lib.fpsk_adjust_logits(s, None, None) == fpsk.ERR_ALIGN


def distill(f, token=P, teacher=P, weight=P, loss=P, lse=P, token_bytes=4, teacher_type=F32, tau=1.0):
    return f(struct.pack("@PPPPPPPqqqqqiiiiiiif", P, token, teacher, weight, loss, lse, P, 100, 4, 4, 100, 2, 100, 4, F32, token_bytes, teacher_type, F32, 1, tau),
             None, None)


def test_distill(lib):
    for f in (lib.fpsk_distill_loss, lib.fpsk_distill_loss_backward):
        assert distill(f, token=P + 2) == distill(f, token=P + 4, token_bytes=8) == distill(f, teacher=P + 2) == fpsk.ERR_ALIGN
        assert distill(f, teacher=P + 1, teacher_type=BF16) == distill(f, weight=P + 2) == distill(f, lse=P + 1) == fpsk.ERR_ALIGN
    assert distill(lib.fpsk_distill_loss, loss=P + 2) == fpsk.ERR_ALIGN
    for f in (lib.fpsk_distill_loss_sums, lib.fpsk_distill_loss_backward_sums):
        f.argtypes = [C.c_void_p] * 4
        assert distill(lambda s, status, stream: f(s, P + 2, status, stream)) == fpsk.ERR_ALIGN
        assert f(None, P, None, None) == fpsk.ERR_NULL
    assert distill(lambda s, status, stream: lib.fpsk_distill_loss_backward_sums(s, None, status, stream), lse=0) == fpsk.ERR_NULL


def test_temperatures_whose_powers_fp32_does_not_hold(lib):
    """1 / tau is representable from 3e-39 on, log2(e) / tau, by which a logit becomes an exponent, from 4.3e-39."""
    for f in (lib.fpsk_distill_loss, lib.fpsk_distill_loss_backward):
        for tau in (3e-39, 4.2e-39):
            assert distill(f, tau=tau) == fpsk.ERR_PARAM
