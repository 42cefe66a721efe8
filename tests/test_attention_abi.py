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
    assert (C.sizeof(A.Rotary), C.sizeof(A.Heads), C.sizeof(A.HeadsGrad)) == (40, 64, 96)
    assert (C.sizeof(A.Cache), C.sizeof(A.Batch), C.sizeof(A.Attention)) == (88, 48, 80)
    assert L.fpsk_norm_rope_workspace_bytes(12) == 0 and L.fpsk_norm_rope_workspace_bytes(128) > 0
    h = A.Heads()
    assert L.fpsk_qk_norm_rope(h, h, 1, 12, 0, 0, None, 0.0, None, None) == fpsk.ERR_SHAPE
    assert L.fpsk_qk_norm_rope(h, h, -1, 16, 0, 0, None, 0.0, None, None) == fpsk.ERR_SHAPE
    assert L.fpsk_qk_norm_rope(h, h, 1, 16, 3, 0, None, 0.0, None, None) == fpsk.ERR_DTYPE
    h.n_heads = 2
    assert L.fpsk_qk_norm_rope(h, None, 1, 16, 0, 0, None, 0.0, None, None) == fpsk.ERR_NULL
    r = A.Rotary()
    r.rot_dim = 24
    assert L.fpsk_qk_norm_rope(None, None, 1, 16, 0, 0, r, 0.0, None, None) == fpsk.ERR_PARAM
    c = A.Cache()
    b = A.Batch()
    assert L.fpsk_paged_append(c, b, h, h, None, 0, None, 0.0, None, None) == fpsk.ERR_NULL
    c.k = c.v = 4096                       # never dereferenced: validation fails first
    c.type, c.n_pages, c.page_size, c.n_heads, c.head_dim = 2, 1, 16, 2, 64
    assert L.fpsk_paged_append(c, b, h, h, None, 0, None, 0.0, None, None) == fpsk.ERR_DTYPE
    c.type = 1
    c.k_page_stride = c.v_page_stride = 2048
    c.k_token_stride = c.v_token_stride = 128
    c.k_head_stride = c.v_head_stride = 32   # heads that overlap
    assert L.fpsk_paged_append(c, b, h, h, None, 0, None, 0.0, None, None) == fpsk.ERR_SHAPE
    c.k_head_stride = c.v_head_stride = 64
    b.n_tokens = 1
    assert L.fpsk_paged_append(c, b, h, h, None, 0, None, 0.0, None, None) == fpsk.ERR_SHAPE   # tokens of no sequence
    b.n_seqs = 1
    assert L.fpsk_paged_append(c, b, h, h, None, 0, None, 0.0, None, None) == fpsk.ERR_NULL
    assert L.fpsk_attention_workspace_init(None, 256, None) == fpsk.ERR_NULL
    assert L.fpsk_attention_workspace_init(C.c_void_p(4097), 256, None) == fpsk.ERR_ALIGN
