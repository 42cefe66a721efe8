"""Automatic differentiation of the operators on a batch without tokens, whose gradients come expanded from a number and are contiguous as they are."""
import pytest
import torch

from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L
from paper_2609_19758_b200 import norm as N

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_tokens(dtype):
    x, residual = (torch.empty(0, 64, dtype=dtype, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.ones(64, device="cuda", requires_grad=True)
    y, h = N.AddRMSNorm.apply(x, residual, w, dtype, 1e-6)
    (y.sum() + h.sum()).backward()
    assert x.grad.shape == residual.grad.shape == (0, 64) and w.grad.shape == (64,) and not bool(w.grad.any())
    z = torch.empty(0, 100, dtype=dtype, device="cuda", requires_grad=True)
    L.DistillLoss.apply(z, torch.empty(0, 4, dtype=torch.int64, device="cuda"), torch.empty(0, 4, device="cuda"), 1.0, True).sum().backward()
    assert z.grad.shape == (0, 100)


def test_no_tokens_in_the_attention_s_norm_and_rotation():
    q, k = (torch.empty(0, heads, 64, dtype=torch.bfloat16, device="cuda", requires_grad=True) for heads in (4, 2))
    qw, kw = (torch.ones(64, device="cuda", requires_grad=True) for _ in range(2))
    cos, sin = A.rotary_tables(16, 64)
    a, b = A.QKNormRope.apply(q, k, qw, kw, cos, sin, torch.empty(0, dtype=torch.int32, device="cuda"), torch.bfloat16, 1e-6, False)
    (a.sum() + b.sum()).backward()
    assert q.grad.shape == (0, 4, 64) and k.grad.shape == (0, 2, 64) and not bool(qw.grad.any()) and not bool(kw.grad.any())
