"""A page number outside the cache reads as a page of zeros, in every form of the attention, and is reported.  Tolerances as in
test_gpu_paged_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

from test_gpu_norm_rope import make_cache
from test_gpu_paged_attention import BF16, F16, UNIT, fill

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("beyond", ["wide", "negative", "no column"])
@pytest.mark.parametrize("seqs,dim,page,dtype,order", [
    ([(1, 200), (1, 100)], 128, 16, BF16, "thd"),
    ([(1, 200), (1, 100)], 128, 16, BF16, "htd"),
    ([(50, 200), (3, 100)], 64, 16, F16, "thd"),         # one tile of queries
    ([(150, 400)], 128, 32, BF16, "thd"),
    ([(30, 200), (1, 100)], 96, 24, F16, "thd"),         # each half of a head by itself
    ([(1, 200), (40, 100)], 128, 12, BF16, "thd"),       # copied by rows
    ([(2, 200), (1, 100)], 256, 16, BF16, "thd"),        # the row kernel
    ([(2, 200), (1, 100)], 256, 12, F16, "htd"),
])
def test_a_page_outside_the_cache_reads_as_zeros(seqs, dim, page, dtype, order, beyond):
    rng = np.random.default_rng(2)
    hq, hk = 4, 2
    k, v, cu, kv, table = make_cache(rng, seqs, hk, dim, page, dtype, order)
    fill(rng, k, v, kv, table, page)
    # the oracle reads a page of zeros of its own
    ko, vo = (torch.cat([t, torch.zeros_like(t[:1])]).double().cpu().numpy() for t in (k, v))
    seen = table.copy()
    if beyond == "no column":                            # more keys than the table has pages for
        columns = int(kv[0]) // page - 2
        seen[0, columns:] = k.shape[0]
        if len(seqs) > 1: seen[1, columns:] = k.shape[0]
        table = table[:, :columns].copy()
    else:
        table[0, 2] = -7 if beyond == "negative" else 12345
        seen[0, 2] = k.shape[0]
    n = int(cu[-1])
    q = torch.from_numpy(rng.standard_normal((n, hq, dim)).astype(np.float32)).to(dtype).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((n, hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_attention(A.PagedCache(k, v), q, out, *(torch.from_numpy(x).cuda() for x in (cu, kv, table)), A.attention_workspace(),
                      max(a for a, _ in seqs), max(b for _, b in seqs), lse=lse, status=status)
    assert int(status) == fpsk.ERR_PARAM
    want, want_lse, mag, smag = O.paged_attention(q.double().cpu().numpy(), ko, vo, cu, kv, seen, dim ** -0.5, True, -1)
    u, e = UNIT[dtype], (dim + 8) * 2.0 ** -23 * smag + 2.0 ** -20
    tol = u * np.abs(want) + mag * (2 * (u + e[..., None]) + 2.0 ** -20) + 2.0 ** -24
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    assert np.all(np.abs(lse.double().cpu().numpy() - want_lse) <= e + 2.0 ** -22 * np.abs(want_lse))
