"""Host-side checks of the attention operators' C ABI that need no GPU: struct layouts and argument validation."""
import ctypes as C

import pytest

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk


@pytest.fixture(scope="module")
def lib():
    B.build()
    return fpsk.lib()


def test_attention_structs_and_validation_need_no_device(lib):
    from paper_2609_19758_b200 import attention as A
    L = A._lib()
    assert (A._ROTARY.size, A._HEADS.size, A._HEADS_GRAD.size) == (40, 64, 96)
    assert (A._CACHE.size, A._BATCH.size, A._ATTENTION.size) == (88, 48, 80)
    assert L.fpsk_norm_rope_workspace_bytes(12) == 0 and L.fpsk_norm_rope_workspace_bytes(128) > 0

    def heads(n):
        return A._HEADS.pack(0, 0, 0, 0, 0, 0, 0, n, 0)

    def rope(q, k=None, n=1, dim=16, types=(0, 0), rot=None, eps=0.0):
        return L.fpsk_qk_norm_rope(q, k, n, dim, types[0], types[1], rot, eps, None, None)

    assert rope(heads(0), heads(0), dim=12) == fpsk.ERR_SHAPE
    assert rope(heads(0), n=-1) == fpsk.ERR_SHAPE
    assert rope(heads(0), types=(3, 0)) == fpsk.ERR_DTYPE
    assert rope(heads(2)) == fpsk.ERR_NULL
    assert rope(None, rot=A._ROTARY.pack(0, 0, 0, 0, 24, 0)) == fpsk.ERR_PARAM
    assert rope(None, eps=-1.0) == fpsk.ERR_PARAM and rope(None, eps=float("nan")) == fpsk.ERR_PARAM

    def append(k=4096, kind=1, head_stride=64, tokens=0, seqs=0):      # the pointer is never read: validation fails first
        c = A._CACHE.pack(k, k, 2048, 128, head_stride, 2048, 128, head_stride, 1, 16, 2, 64, kind)
        b = A._BATCH.pack(0, 0, 0, 0, tokens, seqs, 0)
        return L.fpsk_paged_append(c, b, heads(0), heads(0), None, 0, None, 0.0, None, None)

    assert append(k=0) == fpsk.ERR_NULL
    assert append(kind=2) == fpsk.ERR_DTYPE
    assert append(head_stride=32) == fpsk.ERR_SHAPE                    # heads that overlap
    assert append(tokens=1) == fpsk.ERR_SHAPE                          # tokens of no sequence
    assert append(tokens=1, seqs=1) == fpsk.ERR_NULL
    assert append() == fpsk.ERR_SHAPE                                  # heads of the cache and of k
    assert L.fpsk_attention_workspace_init(None, 256, None) == fpsk.ERR_NULL
    assert L.fpsk_attention_workspace_init(C.c_void_p(4097), 256, None) == fpsk.ERR_ALIGN
