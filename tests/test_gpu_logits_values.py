"""The greedy token and the log-sum-exp of logits whose values stand far apart.  E = 2^-24 is a rounding in FP32."""
import numpy as np
import pytest
import torch

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def test_rows_of_the_lowest_value():
    """Logits that a mask has set to the type's lowest value are numbers still: the first of them is the token, their log-sum-exp that value."""
    for dtype in (F32, BF16, F16):
        low = torch.finfo(dtype).min
        x = torch.full((3, 4001), low, dtype=dtype, device="cuda")
        x[1, 4000] = 1.0
        x[2, 5] = -float("inf")
        token, lse = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
        L.adjust_logits(x, token=token, lse=lse)
        assert token.tolist() == [0, 4000, 0]
        assert lse.tolist()[1] == 1.0
        for r, n in ((0, 4001), (2, 4000)):
            assert float(lse[r]) == pytest.approx(low + np.log(n), rel=4 * E)


@pytest.mark.parametrize("base", [-40.0, -35.0, -28.0])
@pytest.mark.parametrize("vocab", [3000, 3001, 60000])
def test_a_late_largest_costs_no_precision(base, vocab):
    """Three logits near 0 behind a row of others 28 to 40 below.  Their powers have exponents below 4 with the largest as reference: the
    difference (below 2) and the exponent are rounded by 2 E and 2 E ln 2 at most, the power by two units (4 E), sums and joins by some 12 E
    (what is far below the largest adds less than E in all); the logarithm of at most 3 and the sum with the largest by 3 E."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = base + torch.randn(64, vocab, generator=g, device="cuda")
    x = torch.minimum(x, torch.full_like(x, base + 4))
    at = torch.stack([vocab // 2 + torch.randperm(vocab - vocab // 2, generator=g, device="cuda")[:3] for _ in range(64)])
    x.scatter_(1, at, 0.3 * torch.randn(64, 3, generator=g, device="cuda"))
    lse = torch.empty(64, device="cuda")
    L.adjust_logits(x, lse=lse)
    want = torch.logsumexp(x.double(), 1)
    assert float((lse.double() - want).abs().max()) <= 24 * E
