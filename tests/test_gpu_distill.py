"""The loss of logits against a teacher's top logits and its gradient, against the FP64 definitions.

Tolerances: E = 2^-24 is a rounding in FP32.  The log-sum-exp is off by the rounding of its largest term's exponent (2 E of it), of the
powers (2 units) and of the sums (vocab / 512 terms of a lane behind one another or fewer, and 24 joins), relative: together
lse_bound().  The loss adds at most 1024 / 512 terms on a lane and 32 sums of lanes, each of the magnitudes that the oracle
gives: 64 E of them.  A probability is off by the exponent's rounding, E (|y| + |lse|) 1.5, lse's error and two units."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = 2.0 ** -24
TINY = {F32: 2.0 ** -126, F16: 2.0 ** -25, BF16: 2.0 ** -126}          # (powers below 2^-126 are zero)


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def np64(t):
    return t.double().cpu().numpy()


def make(seed, rows, vocab, top, dtype, ttype=F32, token_dtype=torch.int32, pad=0, normalize=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (2.0 * torch.randn(rows, vocab + pad, generator=g, device="cuda")).to(dtype)[:, :vocab]
    token = torch.randint(-1, vocab + 1, (rows, top), generator=g, device="cuda").to(token_dtype)       # some are no tokens, some come twice
    if top > 3:
        token[:, 3] = token[:, 0]
    t = 3.0 * torch.randn(rows, top, generator=g, device="cuda")
    if not normalize:
        t = torch.log_softmax(t, 1) - 0.2 if top else t
    t = t.to(ttype)
    if top > 5:
        t[:, 5] = -float("inf")
    return x, token, t


def lse_bound(x, temperature, vocab):
    x = x[np.isfinite(x)]                                              # (a logit of -inf adds an exact zero)
    return 4 * E * np.abs(x / temperature).max() + (vocab / 64 + 64) * E


def check(x, token, t, temperature, normalize, weight, loss, lse, dlogits):
    raw, tok, tl = np64(x), token.cpu().numpy(), np64(t)
    for i in range(x.shape[0]):
        w = 1.0 if weight is None else float(weight[i])
        if w == 0.0:
            assert (loss is None or float(loss[i]) == 0.0) and (dlogits is None or bool((dlogits[i] == 0).all()))
            continue
        l, dx, s, mag, dmag = D.distill(raw[i], tok[i], tl[i], temperature, normalize)
        off = lse_bound(raw[i], temperature, x.shape[1])
        if lse is not None:
            assert abs(float(lse[i]) - s) <= off
        if loss is not None:
            assert abs(float(loss[i]) - l) <= 64 * E * mag + off * (1 if normalize else np.exp(tl[i][np.isfinite(tl[i])]).sum())
        if dlogits is not None:
            u = torch.finfo(dlogits.dtype).eps / 2
            # the teacher's probabilities: logarithms rounded at their magnitude (at most 64 E of it), 20 or so here
            y = np.where(np.isfinite(raw[i]), np.abs(raw[i] / temperature), 0.0)   # (the probability of -inf is an exact zero)
            rel = off + E * (3 * y + 3 * abs(s) + 1500 + 40)
            assert np.all(np.abs(np64(dlogits[i]) - w * dx) <= u * np.abs(w * dx) + rel * abs(w) * dmag + TINY[dlogits.dtype])


CASES = [(3, 1, 1, F32, F32, F32, 0, 1.0, True), (2, 5, 9, F32, F16, F16, 0, 2.0, True), (4, 1000, 0, F32, F32, BF16, 0, 1.0, True),
         (5, 4096, 64, BF16, BF16, BF16, 0, 1.0, False), (3, 4097, 100, F16, F32, F16, 3, 0.5, True), (300, 2051, 7, F32, F32, BF16, 0, 1.0, True),
         (2, 50257, 1024, F16, F32, F16, 0, 1.5, True), (1, 131072, 32, F32, F32, BF16, 0, 1.0, True), (2, 131072, 600, BF16, F16, F32, 0, 3.0, True),
         (160, 32000, 20, F32, F32, F32, 0, 1.0, False), (1, 400001, 10, F32, F32, F32, 0, 1.0, True), (1, 1000003, 10, BF16, F32, BF16, 0, 1.0, True)]


@pytest.mark.parametrize("rows,vocab,top,src,ttype,grad,pad,temperature,normalize", CASES)
def test_loss_and_gradient(rows, vocab, top, src, ttype, grad, pad, temperature, normalize):
    x, token, t = make(vocab, rows, vocab, top, src, ttype, torch.int64 if vocab % 2 else torch.int32, pad, normalize)
    before = x.clone()
    how = dict(temperature=temperature, normalize=normalize)
    weight = 0.25 + torch.rand(rows, device="cuda")
    if rows > 2:
        weight[1] = 0.0
    loss, lse = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    dx = torch.full((rows, vocab + pad), 7.0, dtype=grad, device="cuda")
    L.distill_loss(x, token, t, loss, row_weight=weight, lse=lse, dlogits=dx[:, :vocab], **how)
    check(x, token, t, temperature, normalize, weight, loss, lse, dx[:, :vocab])
    assert bool((dx[:, vocab:] == 7.0).all()) and torch.equal(x, before)
    # the loss alone, without weights
    alone, lse1 = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    L.distill_loss(x, token, t, alone, lse=lse1, **how)
    check(x, token, t, temperature, normalize, None, alone, lse1, None)
    # the gradient alone
    back = torch.full((rows, vocab + pad), 7.0, dtype=grad, device="cuda")
    L.distill_loss_backward(x, token, t, lse1, weight, back[:, :vocab], **how)
    check(x, token, t, temperature, normalize, weight, None, None, back[:, :vocab])
    assert bool((back[:, vocab:] == 7.0).all())
    if src == grad:
        kept, l2 = dx[:, :vocab].clone(), torch.empty_like(loss)
        y = x.clone()
        L.distill_loss(y, token, t, l2, row_weight=weight, dlogits=y, **how)                             # in place
        assert torch.equal(y, kept) and torch.equal(l2, loss)
        y = x.clone()
        L.distill_loss_backward(y, token, t, lse1, weight, y, **how)
        assert torch.equal(y, back[:, :vocab])


def test_rows_without_a_teacher_and_rows_without_weight():
    x, token, t = make(1, 6, 3000, 8, F32)
    x[0] = float("nan")                                                # of weight 0: not read
    t[0] = float("nan")
    token[1] = -1
    t[2] = -float("inf")
    x[3] = float("nan")                                                # no teacher, so that nothing of it reaches the loss
    token[3] = 3000
    x[4, 100:] = -float("inf")
    token[4] = torch.arange(8, device="cuda")
    t[4] = torch.arange(8, device="cuda").float()
    weight = torch.ones(6, device="cuda")
    weight[0] = 0.0
    loss, dx = torch.full((6,), 7.0, device="cuda"), torch.full((6, 3000), 7.0, device="cuda")
    L.distill_loss(x, token, t, loss, row_weight=weight, dlogits=dx)
    assert loss[:4].tolist() == [0.0] * 4 and bool((dx[:4] == 0).all())
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(dx).all()) and bool((dx[4, 100:] == 0).all())
    check(x[4:], token[4:], t[4:], 1.0, True, None, loss[4:], None, dx[4:])
    # a listed token that the student holds impossible
    x[5, 7] = -float("inf")
    token[5] = torch.tensor([7, 8, 9, 10, 11, 12, 13, 14], device="cuda")
    t[5] = 0.0
    L.distill_loss(x, token, t, loss, row_weight=weight, dlogits=dx)
    assert float(loss[5]) == float("inf") and float(dx[5, 7]) == pytest.approx(-0.125, rel=64 * E) and bool(torch.isfinite(dx[5]).all())


def test_far_logits():
    """Scores of large magnitude, and one that stands out by more than the powers' range."""
    x, token, t = make(2, 4, 5000, 6, F32)
    x[0] += 3e4
    x[1] -= 3e4
    x[2, 17] = 500.0
    x[3] *= 40.0
    loss, dx = torch.empty(4, device="cuda"), torch.empty(4, 5000, device="cuda")
    L.distill_loss(x, token, t, loss, dlogits=dx)
    check(x, token, t, 1.0, True, None, loss, None, dx)


def test_gradient_against_differences():
    """The loss's own differences: a step of 2^-4 is off by its third derivative (at most step^2 / 6 of a probability) and by the
    losses' roundings."""
    x, token, t = make(3, 1, 200, 12, F32)
    dx, loss = torch.empty(1, 200, device="cuda"), torch.empty(1, device="cuda")
    L.distill_loss(x, token, t, loss, dlogits=dx, temperature=1.5)
    step, n = 2.0 ** -4, 200
    up, down = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    for sign, out in ((1, up), (-1, down)):
        L.distill_loss(x + sign * step * torch.eye(n, device="cuda"), token.expand(n, 12).contiguous(), t.expand(n, 12).contiguous(), out, temperature=1.5)
    got = (up - down) / (2 * step)
    _, _, lse, mag, _ = D.distill(np64(x)[0], token[0].tolist(), np64(t)[0], 1.5, True)
    bound = step ** 2 / 6 / 1.5 ** 3 * 0.2 + 2 * (64 * E * mag + lse_bound(np64(x), 1.5, n)) / (2 * step)
    assert float((got - dx[0]).abs().max()) <= bound


@pytest.mark.parametrize("dtype,normalize", [(F32, True), (BF16, False)])
def test_autograd(dtype, normalize):
    x, token, t = make(4, 9, 3001, 20, dtype, normalize=normalize)
    x = x.clone().requires_grad_()
    w = torch.rand(9, device="cuda")
    loss = L.DistillLoss.apply(x, token, t, 1.3, normalize)
    (loss * w).sum().backward()
    assert x.grad.dtype == dtype
    check(x.detach(), token, t, 1.3, normalize, None, loss.detach(), None, None)
    check(x.detach(), token, t, 1.3, normalize, w, None, None, x.grad)
    x.grad = None
    L.DistillLoss.apply(x, token, t, 1.3, normalize).sum().backward()  # (an expanded gradient)
    check(x.detach(), token, t, 1.3, normalize, None, None, None, x.grad)


def test_repeatable_captured_and_on_another_stream():
    for rows, vocab, dtype in ((3, 131072, F32), (700, 5003, BF16)):
        x, token, t = make(5, rows, vocab, 50, dtype)

        def call(stream=None):
            o = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, vocab, dtype=BF16, device="cuda"), torch.empty(rows, vocab, dtype=BF16, device="cuda")
            one = torch.ones(rows, device="cuda")
            return o, lambda: (L.distill_loss(x, token, t, o[0], lse=o[1], dlogits=o[2], stream=stream), L.distill_loss_backward(x, token, t, o[1], one, o[3], stream=stream))

        first, f = call()
        f()
        again, f = call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        graph.replay()
        st = torch.cuda.Stream()
        third, f = call(st)
        torch.cuda.synchronize()
        f()
        st.synchronize()
        for a, b, c in zip(first, again, third):
            assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("vocab", [700, 5000, 131072])
@pytest.mark.parametrize("grad", [None, F32, BF16])
def test_a_learnt_token_costs_no_precision(vocab, grad):
    """One listed logit stands 40 to 60 above the others: the loss is ln(1 + sum e^(x_v - x_0)), below 1e-12.  Its exponent is 0 when it is the
    reference, and S then 1 with two units of the power and one rounding of a sum or a logarithm each: 2^-23 (2 + 1) at the most.  With
    another logit as reference the exponent, up to 86 in powers of two, is rounded by up to 2^-18."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(64, vocab, generator=g, device="cuda")
    token = torch.randint(0, vocab, (64, 1), generator=g, device="cuda", dtype=torch.int32)
    x.scatter_(1, token.long(), 45.0 + 15.0 * torch.rand(64, 1, generator=g, device="cuda"))
    loss, dx = torch.empty(64, device="cuda"), None if grad is None else torch.empty(64, vocab, device="cuda", dtype=grad)
    L.distill_loss(x, token, torch.zeros(64, 1, device="cuda"), loss, dlogits=dx)
    assert float(loss.abs().max()) <= 3 * 2.0 ** -23


def test_no_rows():
    x = torch.empty(0, 100, device="cuda")
    L.distill_loss(x, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, 4, device="cuda"), torch.empty(0, device="cuda"), dlogits=torch.empty_like(x))


def test_refusals():
    x, token, t = make(6, 3, 100, 4, F32)
    loss, dx = torch.full((3,), 7.0, device="cuda"), torch.full((3, 100), 7.0, device="cuda")
    for bad in (lambda: L.distill_loss(x, token[:2], t, loss), lambda: L.distill_loss(x, token, t[:, :3], loss), lambda: L.distill_loss(x, token, t, loss[:2]),
                lambda: L.distill_loss(x, token, t, loss, dlogits=dx[:, :99]), lambda: L.distill_loss(x, token, t, loss, dlogits=dx[:1].expand(3, 100)),
                lambda: L.distill_loss(x, token, t, loss, temperature=0.0), lambda: L.distill_loss(x, token, t, loss, temperature=-1.0),
                lambda: L.distill_loss(x, token, t, loss, temperature=float("inf")), lambda: L.distill_loss(x, token, t, loss, temperature=float("nan")),
                lambda: L.distill_loss(x, token, t, loss, row_weight=loss.half()), lambda: L.distill_loss(x.t(), token, t, loss), lambda: L.distill_loss(x, token.cpu(), t, loss)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: L.distill_loss(x.double(), token, t, loss), lambda: L.distill_loss(x, token.short(), t, loss), lambda: L.distill_loss(x, token, t.double(), loss),
                lambda: L.distill_loss(x, token, t, loss, temperature="1")):
        with pytest.raises(TypeError):
            bad()
    many = torch.zeros(3, 1025, dtype=torch.int32, device="cuda")
    for bad in (lambda: L.distill_loss(x, many, many.float(), loss), lambda: L.distill_loss(x, token, t, None), lambda: L.distill_loss_backward(x, token, t, None, loss, dx),
                lambda: L.distill_loss_backward(x, token, t, loss, loss, None)):
        with pytest.raises(RuntimeError):
            bad()
    assert bool((loss == 7.0).all()) and bool((dx == 7.0).all())
