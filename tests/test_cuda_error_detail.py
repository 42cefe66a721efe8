"""A failed CUDA call is named: the error, the source line and the call.  On a machine without a device every call into CUDA fails,
which needs no fault to be made."""
import ctypes as C
import threading

import pytest
import torch

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="CUDA calls succeed here")


@pytest.fixture(scope="module")
def lib():
    B.build()
    return fpsk.lib()


def test_the_error_its_place_and_its_call(lib):
    memory = C.create_string_buffer(1024)
    at = (C.addressof(memory) + 255) & ~255
    assert lib.fpsk_probe_init(at, 256, None) == fpsk.ERR_CUDA          # no device: the memset is refused on the host
    detail = fpsk.last_cuda_error()
    assert detail.startswith("cudaError") and "api.cu:" in detail and "cudaMemsetAsync" in detail
    assert detail in str(fpsk.FpskError(fpsk.ERR_CUDA, "fpsk_probe_init"))
    assert detail not in str(fpsk.FpskError(fpsk.ERR_SHAPE, "fpsk_probe_init"))
    seen = []
    other = threading.Thread(target=lambda: seen.append(fpsk.last_cuda_error()))
    other.start()
    other.join()
    assert seen == [""]                                              # each thread has its own


def test_other_files_and_contexts_name_theirs(lib):
    out = C.c_void_p()
    assert lib.fpsk_context_create(C.byref(out)) == fpsk.ERR_CUDA and not out.value
    assert "sketch.cu:" in fpsk.last_cuda_error()
