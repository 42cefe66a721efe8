"""The loss against a teacher where the kernel goes on from row to row, and where a listed token has been learnt.  E = 2^-24 is a rounding in FP32."""
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


def listed(seed, rows, vocab, top, dtype, normalize):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (2.0 * torch.randn(rows, vocab, generator=g, device="cuda")).to(dtype)
    token = torch.randint(-1, vocab + 1, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    if top > 3:
        token[::2, 3] = token[::2, 0]                                  # listed twice, in half of the rows
    t = 3.0 * torch.randn(rows, top, generator=g, device="cuda")
    if not normalize:
        t = torch.log_softmax(t, 1) - 0.2
    weight = 0.25 + torch.rand(rows, generator=g, device="cuda")
    weight[torch.rand(rows, generator=g, device="cuda") < 0.3] = 0.0
    token[torch.rand(rows, generator=g, device="cuda") < 0.05] = -1    # rows without a teacher
    return x, token, t, weight


@pytest.mark.parametrize("rows,vocab,top,dtype,grad", [
    (2500, 3001, 20, F32, F32), (2500, 3000, 400, F32, BF16), (2500, 3002, 161, BF16, F32), (700, 40001, 20, F32, F32), (700, 40000, 600, F16, F16),
    (1000, 131072, 200, BF16, BF16)])
@pytest.mark.parametrize("normalize", [True, False])
def test_many_rows_of_a_cluster(rows, vocab, top, dtype, grad, normalize):
    """More rows than clusters fit the device, weights of 0 and rows without a teacher between them, one warp of the teacher and three: rings,
    double buffers, lists and maps are used for one row after another."""
    x, token, t, weight = listed(vocab + top, rows, vocab, top, dtype, normalize)
    how = dict(temperature=1.5, normalize=normalize)
    few = slice(None) if rows * vocab < 1e8 else slice(0, rows, 7)     # (the oracle's time)
    loss, lse, dx = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda"), torch.full((rows, vocab), 7.0, dtype=grad, device="cuda")
    L.distill_loss(x, token, t, loss, row_weight=weight, lse=lse, dlogits=dx, **how)
    check(x[few], token[few], t[few], 1.5, normalize, weight[few], loss[few], lse[few], dx[few])
    back = torch.full_like(dx, 7.0)
    L.distill_loss_backward(x, token, t, lse, weight, back, **how)
    check(x[few], token[few], t[few], 1.5, normalize, weight[few], None, None, back[few])
    alone, lse1 = torch.full_like(loss, 7.0), torch.full_like(loss, 7.0)
    L.distill_loss(x, token, t, alone, row_weight=weight, lse=lse1, **how)
    check(x[few], token[few], t[few], 1.5, normalize, weight[few], alone[few], lse1[few], None)
    # every row, not the oracle's alone: each form has the others' values to the bounds of both
    live = weight != 0
    assert float((loss - alone)[live].abs().max()) <= 1e-4 and bool((loss[~live] == 0).all()) and bool((dx[~live] == 0).all()) and bool((back[~live] == 0).all())
    u = 2 * torch.finfo(grad).eps
    assert bool(((dx.float() - back.float()).abs() <= u * dx.float().abs() + 1e-4 * weight[:, None]).all())
    if dtype == grad:
        y, l2 = x.clone(), torch.empty_like(loss)
        L.distill_loss(y, token, t, l2, row_weight=weight, dlogits=y, **how)
        assert torch.equal(y, dx) and torch.equal(l2, loss)
        y = x.clone()
        L.distill_loss_backward(y, token, t, lse, weight, y, **how)
        assert torch.equal(y, back)


@pytest.mark.parametrize("vocab", [700, 5001, 131072])
@pytest.mark.parametrize("grad", [F32, BF16])
def test_gradients_of_a_learnt_token(vocab, grad):
    """A listed logit 12 to 20 above the others beside a second listed one among them: gradients and the loss, which is not 0, by the bounds of
    the outliers' test (the teacher's probabilities: |t| below 8, 20 E more)."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 64
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    token = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:2] for _ in range(rows)]).to(torch.int32)
    x.scatter_(1, token[:, :1].long(), 12.0 + 8.0 * torch.rand(rows, 1, generator=g, device="cuda"))
    t = torch.tensor([[6.0, 0.5]], device="cuda").repeat(rows, 1)
    loss, dx = torch.empty(rows, device="cuda"), torch.empty(rows, vocab, dtype=grad, device="cuda")
    L.distill_loss(x, token, t, loss, dlogits=dx)
    u = torch.finfo(grad).eps / 2
    for i in range(rows):
        raw = np64(x[i])
        l, d, _, mag, dmag = D.distill(raw, token[i].tolist(), t[i].tolist(), 1.0, True)
        assert l > 1e-3 and abs(float(loss[i]) - l) <= 64 * E * mag
        assert np.all(np.abs(np64(dx[i]) - d) <= u * np.abs(d) + (70 + 2 * (raw.max() - raw)) * E * dmag + 2.0 ** -126)


def test_padding_in_autograd():
    """Rows without weight hold NaN and infinities, which reach neither the weighted sum nor the gradient."""
    x, token, t, weight = listed(9, 300, 4001, 12, F32, True)
    pad = weight == 0
    x[pad] = float("nan")
    x[pad.nonzero()[0]] = float("inf")
    t[pad] = float("nan")
    assert 50 < int(pad.sum()) < 150
    x.requires_grad_()
    loss = L.DistillLoss.apply(x, token, t, 1.0, True, weight)
    (loss * weight).sum().backward()
    check(x.detach(), token, t, 1.0, True, weight, loss.detach(), None, x.grad)
    x.grad = None
    L.DistillLoss.apply(x, token, t, 1.0, True, weight).sum().backward()                 # (whatever gradient a loss of padding gets)
    check(x.detach(), token, t, 1.0, True, (~pad).float(), None, None, x.grad)
    # as before without it
    y = x.detach()[~pad].requires_grad_()
    L.DistillLoss.apply(y, token[~pad], t[~pad], 1.0, True).sum().backward()
    check(y.detach(), token[~pad], t[~pad], 1.0, True, None, None, None, y.grad)
