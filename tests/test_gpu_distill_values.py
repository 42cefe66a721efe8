"""The loss against a teacher and its gradient where values stand far apart: wide vocabularies, masked entries, outliers, lowest values, shifted
rows, and temperatures at the ends of their range, against the FP64 definitions.  E = 2^-24 is a rounding in FP32."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L
from test_gpu_distill import check, np64

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("rows,vocab,top", [(450, 1600000, 64), (450, 1500000, 1024), (230, 3100000, 8), (120, 6200000, 8), (2, 1 << 23, 1024)])
def test_the_gradient_alone_of_wide_vocabularies(rows, vocab, top):
    """Enough rows for the SMs with one block each or two, and more tokens than the map of so few blocks holds."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    live = torch.tensor([0, rows // 2, rows - 1], device="cuda")
    x = torch.zeros(rows, vocab, dtype=F16, device="cuda")
    for r in live.tolist():
        x[r].normal_(generator=g)
    token = torch.randint(0, vocab, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    token[:, -1] = vocab - 1
    t = torch.randn(rows, top, generator=g, device="cuda")
    weight = torch.zeros(rows, device="cuda")
    weight[live] = 1024.0
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    L.distill_loss(x, token, t, loss, row_weight=weight, lse=lse)
    dx = torch.full_like(x, 7.0)
    L.distill_loss_backward(x, token, t, lse, weight, dx)
    check(x[live], token[live], t[live], 1.0, True, weight[live], loss[live], lse[live], dx[live])
    del x
    dx[live] = 0.0
    assert not bool(dx.any())
