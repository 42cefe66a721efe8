"""Attention over pages of many sequences: more than a block's threads, as many as its table of work holds, and one more.  Tolerances as
in test_gpu_paged_attention.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B

from test_gpu_paged_attention import BF16, F16, UNIT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def lengths(n, new, keys, seed):
    """New tokens and keys of n sequences, among them ones of none."""
    rng = np.random.default_rng(seed)
    q = rng.integers(0, new + 1, n)
    k = np.maximum(rng.integers(0, keys + 1, n), q)
    k[rng.random(n) < 0.1] = 0                   # tokens without a place
    return q.astype(np.int32), k.astype(np.int32)


@pytest.mark.parametrize("n,new,keys,hq,hk,dim,page,dtype", [
    (384, 1, 60, 2, 1, 128, 16, BF16),           # as many as threads
    (385, 1, 60, 2, 1, 128, 16, BF16),
    (1000, 2, 200, 4, 2, 128, 16, BF16),
    (1000, 2, 200, 4, 2, 128, 12, F16),          # copied by rows
    (769, 40, 90, 1, 1, 64, 16, F16),            # a tile of queries each
    (500, 30, 300, 2, 2, 128, 8, BF16),          # two tiles each
    (1153, 1, 40, 2, 1, 256, 16, BF16),          # the row kernel
    (16384, 1, 20, 2, 1, 64, 8, BF16),           # the whole table of work
    (16384, 1, 20, 2, 1, 128, 8, F16),
    (16385, 1, 20, 2, 1, 64, 8, BF16),           # one more: the row kernel
])
def test_many_sequences(n, new, keys, hq, hk, dim, page, dtype):
    rng = np.random.default_rng(n + dim)
    ql, kl = lengths(n, new, keys, n)
    cu = np.concatenate([[0], np.cumsum(ql)]).astype(np.int32)
    pages = -(-kl // page)
    total = int(pages.sum()) + 3
    k, v = (torch.from_numpy(rng.standard_normal((total, page, hk, dim)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    table = np.full((n, int(pages.max())), -1, dtype=np.int32)
    order, at = rng.permutation(total), 0
    for b, c in enumerate(pages):
        table[b, :c] = order[at:at + c]
        at += c
    q = torch.from_numpy(rng.standard_normal((int(cu[-1]), hq, dim)).astype(np.float32)).to(dtype).cuda()
    out, lse = torch.full_like(q, 7.0), torch.full((int(cu[-1]), hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_attention(A.PagedCache(k, v), q, out, *(torch.from_numpy(x).cuda() for x in (cu, kl, table)), A.attention_workspace(), new, keys,
                      lse=lse, status=status)
    assert int(status) == 0
    want, want_lse, mag, smag = O.paged_attention(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(), cu, kl, table,
                                                  dim ** -0.5, True, -1)
    u, e = UNIT[dtype], (dim + 8) * 2.0 ** -23 * smag + 2.0 ** -20
    tol = u * np.abs(want) + mag * (2 * (u + e[..., None]) + 2.0 ** -20) + 2.0 ** -24
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    none, got = np.isneginf(want_lse), lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got), none)
    assert np.all(np.abs(got[~none] - want_lse[~none]) <= e[~none] + 2.0 ** -22 * np.abs(want_lse[~none]))
