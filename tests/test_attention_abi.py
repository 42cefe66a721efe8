"""Host-side checks of the attention operators' C ABI that need no GPU: struct layouts and argument validation."""
import ctypes as C
import struct

import pytest

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk


@pytest.fixture(scope="module")
def lib():
    B.build()
    return fpsk.lib()


def test_attention_structs_and_validation_need_no_device(lib):
    # the header's structs, as a foreign caller would lay them out
    HEADS, ROTARY, CACHE, BATCH = (struct.Struct(f) for f in ("@PPPqqqqii", "@PPPqii", "@PPqqqqqqqiiii", "@PPPqqii"))
    L = lib
    vp, i64, i32 = C.c_void_p, C.c_int64, C.c_int32
    L.fpsk_qk_norm_rope.argtypes = [vp, vp, i64, i32, C.c_int, C.c_int, vp, C.c_float, vp, vp]
    L.fpsk_paged_append.argtypes = [vp, vp, vp, vp, vp, C.c_int, vp, C.c_float, vp, vp]
    L.fpsk_norm_rope_workspace_bytes.argtypes, L.fpsk_norm_rope_workspace_bytes.restype = [i32], C.c_size_t
    L.fpsk_attention_workspace_init.argtypes = [vp, C.c_size_t, vp]
    assert L.fpsk_norm_rope_workspace_bytes(12) == 0 and L.fpsk_norm_rope_workspace_bytes(128) > 0

    def heads(n):
        return HEADS.pack(0, 0, 0, 0, 0, 0, 0, n, 0)

    def rope(q, k=None, n=1, dim=16, types=(0, 0), rot=None, eps=0.0):
        return L.fpsk_qk_norm_rope(q, k, n, dim, types[0], types[1], rot, eps, None, None)

    assert rope(heads(0), heads(0), dim=12) == fpsk.ERR_SHAPE
    assert rope(heads(0), n=-1) == fpsk.ERR_SHAPE
    assert rope(heads(0), types=(3, 0)) == fpsk.ERR_DTYPE
    assert rope(heads(2)) == fpsk.ERR_NULL
    assert rope(None, rot=ROTARY.pack(0, 0, 0, 0, 24, 0)) == fpsk.ERR_PARAM
    assert rope(None, eps=-1.0) == fpsk.ERR_PARAM and rope(None, eps=float("nan")) == fpsk.ERR_PARAM

    def append(k=4096, kind=1, head_stride=64, tokens=0, seqs=0):      # the pointer is never read: validation fails first
        c = CACHE.pack(k, k, 2048, 128, head_stride, 2048, 128, head_stride, 1, 16, 2, 64, kind)
        b = BATCH.pack(0, 0, 0, 0, tokens, seqs, 0)
        return L.fpsk_paged_append(c, b, heads(0), heads(0), None, 0, None, 0.0, None, None)

    assert append(k=0) == fpsk.ERR_NULL
    assert append(kind=2) == fpsk.ERR_DTYPE
    assert append(head_stride=32) == fpsk.ERR_SHAPE                    # heads that overlap
    assert append(tokens=1) == fpsk.ERR_SHAPE                          # tokens of no sequence
    assert append(tokens=1, seqs=1) == fpsk.ERR_NULL
    assert append() == fpsk.ERR_SHAPE                                  # heads of the cache and of k
    assert L.fpsk_attention_workspace_init(None, 256, None) == fpsk.ERR_NULL
    assert L.fpsk_attention_workspace_init(C.c_void_p(4097), 256, None) == fpsk.ERR_ALIGN


def test_binding_refuses_tensors_of_the_host():
    import torch
    from paper_2609_19758_b200 import attention as A
    x = torch.zeros(2, 3, 16)
    with pytest.raises(ValueError):
        A.qk_norm_rope(x, None, None, None, None, x.clone(), None)
    with pytest.raises(ValueError):
        A.PagedCache(torch.zeros(2, 4, 1, 16, dtype=torch.float16), torch.zeros(2, 4, 1, 16, dtype=torch.float16))
    with pytest.raises(TypeError):
        A.qk_norm_rope("q", None, None, None, None, x, None)
