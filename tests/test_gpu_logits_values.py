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
