"""The loss against a teacher and its gradient where values stand far apart: wide vocabularies, masked entries, outliers, lowest values, shifted
rows, and temperatures at the ends of their range, against the FP64 definitions.  E = 2^-24 is a rounding in FP32."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L
from test_gpu_distill import check, lse_bound, np64

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


@pytest.mark.parametrize("top", [1, 8, 100, 600])
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("ttype,low", [(F32, -1e9), (F32, -1e30), (F16, -65504.0), (BF16, -1e4)])
def test_listed_entries_that_a_finite_number_masks(top, normalize, ttype, low):
    """Entries that a mask has set to a large negative number add nothing, wherever they stand in the list, and whatever the student's logit
    of them is; the others keep their precision (the bounds of `test_gpu_distill.check` for the logits that are not masked)."""
    g = torch.Generator(device="cuda").manual_seed(top)
    rows, vocab = 12, 5003
    x = 2.0 * torch.randn(rows, vocab, generator=g, device="cuda")
    token = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:top] for _ in range(rows)]).to(torch.int32)
    t = 2.0 * torch.randn(rows, top, generator=g, device="cuda")
    if not normalize:
        t = torch.log_softmax(t, 1) - 0.1
    t = t.to(ttype)
    kept = t.clone()
    t[:4, 0] = low
    t[4:8, :top // 2] = low
    t[8:10, :max(top - 1, 0)] = low                                    # the last one counts
    t[10, ::2] = low
    t[11] = low                                                        # all of them: as likely as each other, or (as given) not at all
    if top == 600:
        t[8, :] = low
        t[8, 450] = kept[8, 450]
    # half of the rows: the student's logits of those tokens masked as well
    for r in range(0, rows - 1, 2):
        x[r, token[r][t[r] == low].long()] = -1e9
    loss, lse, dx = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    L.distill_loss(x, token, t, loss, lse=lse, dlogits=dx, normalize=normalize, temperature=1.25)
    alone = torch.empty_like(loss)
    L.distill_loss(x, token, t, alone, normalize=normalize, temperature=1.25)
    for r in range(rows):
        raw, tl = np64(x[r]), np64(t[r])
        if normalize and np.all(tl == tl[0]) and tl[0] < -1e3:
            tl = np.zeros(top)                                         # (the same row, where 64 bits hold its logarithms and the bounds are not the mask's size)
        l, d, s, mag, dmag = D.distill(raw, token[r].tolist(), tl, 1.25, normalize)
        off = lse_bound(raw[raw > -1e8], 1.25, vocab)
        mass = 1.0 if normalize else np.exp(tl).sum()
        assert abs(float(lse[r]) - s) <= off
        assert max(abs(float(loss[r]) - l), abs(float(alone[r]) - l)) <= 64 * E * mag + off * mass
        y = np.where(raw > -1e8, np.abs(raw / 1.25), 0.0)
        assert np.all(np.abs(np64(dx[r]) - d) <= (off + E * (3 * y + 3 * abs(s) + 1540)) * dmag + 2.0 ** -126)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_of_the_types_lowest_value(dtype):
    """A mask of the type's lowest value over everything leaves tokens that are as likely as each other."""
    rows, vocab, top = 3, 3001, 9
    low = torch.finfo(dtype).min
    x = torch.full((rows, vocab), low, dtype=dtype, device="cuda")
    x[1, 77] = 0.5                                                     # but one
    token = torch.arange(70, 70 + top, device="cuda", dtype=torch.int32).repeat(rows, 1)
    t = torch.randn(rows, top, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    t[1] = -float("inf")
    t[1, 7] = 2.0
    t[2] = torch.finfo(F32).min                                        # the teacher's as well
    loss, dx = torch.empty(rows, device="cuda"), torch.empty(rows, vocab, device="cuda")
    L.distill_loss(x, token, t, loss, dlogits=dx)
    p = torch.softmax(t.double(), 1)
    p[2] = 1.0 / top
    want = torch.full((rows, vocab), 1.0 / vocab, dtype=torch.float64, device="cuda")
    want[1] = 0.0
    want[1, 77] = 1.0
    want.scatter_add_(1, token.long(), -p)
    # powers of 0 are 1: a rounding for each of some 16 sums and 24 joins, a product, a quotient
    assert float((dx.double() - want).abs().max()) <= 64 * E
    held = np.log(vocab) + (torch.special.xlogy(p, p)).sum(1)
    held[1] = 0.0
    assert float((loss.double() - held).abs().max()) <= 64 * E * 10


@pytest.mark.parametrize("rows,vocab", [(128, 5000), (128, 5003), (24, 131072), (600, 20001)])
@pytest.mark.parametrize("temperature", [1.0, 0.5])
def test_an_outlier_that_is_not_listed_costs_no_precision(rows, vocab, temperature):
    """One logit 30 to 50 (in units of the temperature) above the others, anywhere in the row, first and last elements among them.

    A power 2^y with |y| <= 8 is off by the difference x - M (below 8 temperatures: 4 E of the power), by y's own rounding (4 E ln 2) and by the
    powers' two units (4 E); the sum as much, and by 16 roundings of additions and joins; the factor by 5 roundings: 48 E.  A logit d
    below the largest: its exponent is rounded at its size, twice: 2 d E more.  The teacher's probabilities are equal (2 E)."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    at = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    at[:8] = torch.tensor([0, 1, 2, 3, vocab - 1, vocab - 2, vocab - 3, vocab - 4], device="cuda")
    x[torch.arange(rows, device="cuda"), at] = 30.0 + 20.0 * torch.rand(rows, generator=g, device="cuda")
    x *= temperature
    token = torch.randint(0, vocab, (rows, 6), generator=g, device="cuda", dtype=torch.int32)
    t = torch.zeros(rows, 6, device="cuda")
    loss, dx = torch.empty(rows, device="cuda"), torch.empty_like(x)
    L.distill_loss(x, token, t, loss, dlogits=dx, temperature=temperature)
    for i in range(rows):
        _, d, lse, _, mag = D.distill(np64(x[i]), token[i].tolist(), [0.0] * 6, temperature, True)
        below = (np64(x[i]).max() - np64(x[i])) / temperature
        assert np.all(np.abs(np64(dx[i]) - d) <= (50 + 2 * below) * E * mag + 2.0 ** -126), i


@pytest.mark.parametrize("shift", [0.0, 300.0, -5000.0])
@pytest.mark.parametrize("normalize", [True, False])
def test_autograd_does_not_round_at_the_logarithms_size(shift, normalize):
    """The gradient of DistillLoss for rows whose log-sum-exp is large, as exact as that of the fused call: the bounds of the outliers' test
    without an outlier, with 40 E more for p = e^t of t between -20 and 0, twice rounded."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, vocab = 40, 20003
    x = (2.0 * torch.randn(rows, vocab, generator=g, device="cuda") + shift).requires_grad_()
    token = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:12] for _ in range(rows)])
    t = 2.0 * torch.randn(rows, 12, generator=g, device="cuda")
    if not normalize:
        t = torch.log_softmax(t, 1) - 0.1
    w = torch.rand(rows, generator=g, device="cuda")
    w[3] = 0.0
    (L.DistillLoss.apply(x, token, t, 1.0, normalize) * w).sum().backward()
    fused, loss = torch.empty(rows, vocab, device="cuda"), torch.empty(rows, device="cuda")
    L.distill_loss(x.detach(), token, t, loss, row_weight=w, dlogits=fused, normalize=normalize)
    for i in range(rows):
        raw = np64(x.detach()[i])
        _, d, _, _, mag = D.distill(raw, token[i].tolist(), t[i].tolist(), 1.0, normalize)
        for got in (x.grad[i], fused[i]):
            assert np.all(np.abs(np64(got) - float(w[i]) * d) <= float(w[i]) * (90 + 2 * (raw.max() - raw)) * E * mag + 2.0 ** -126), i


def test_sums_that_are_refused_and_rows_without_weight():
    x, token, t = torch.randn(3, 500, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda"), torch.zeros(3, 2, device="cuda")
    loss, dx, weight = torch.empty(3, device="cuda"), torch.empty(3, 500, device="cuda"), torch.tensor([1.0, 0.0, 1.0], device="cuda")
    sums = torch.full((3, 2), 7.0, device="cuda")
    for bad in (sums[:2], sums[:, :1], sums.double(), sums.t().contiguous().t(), torch.zeros(3, 4, device="cuda")[:, :2], sums.cpu()):
        with pytest.raises(ValueError):
            L.distill_loss(x, token, t, loss, sums=bad)
    with pytest.raises(RuntimeError):
        L.distill_loss_backward(x, token, t, None, loss, dx)           # neither sums nor lse
    assert bool((sums == 7.0).all())
    lse = torch.empty(3, device="cuda")
    L.distill_loss(x, token, t, loss, row_weight=weight, lse=lse, sums=sums)
    assert sums[1].tolist() == [0.0, 1.0] and float(lse[1]) == 0.0
    assert float((sums[:, 0] + sums[:, 1].log() - lse).abs().max()) <= 4 * E * 10
    L.distill_loss_backward(x, token, t, None, weight, dx, sums=sums)
    check(x, token, t, 1.0, True, weight, loss, lse, dx)
    empty = torch.empty(0, 500, device="cuda")
    L.distill_loss(empty, token[:0], t[:0], loss[:0], sums=sums[:0])


def test_the_highest_temperatures():
    """The log-sum-exp times the temperature is beyond FP32, its powers are not.  A factor of 1 / temperature below the normal numbers is off by
    2^-149 / 1e-38, twice."""
    x = torch.randn(4, 5001, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    token = torch.arange(8, device="cuda", dtype=torch.int32).repeat(4, 1)
    t = torch.zeros(4, 8, device="cuda")
    weight = torch.full((4,), 1e30, device="cuda")
    want = torch.full((4, 5001), 1.0 / 5001, dtype=torch.float64, device="cuda")
    want[:, :8] -= 0.125
    for tau in (1e6, 1e37, 1e38):
        loss, lse, dx, back = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(x), torch.empty_like(x)
        L.distill_loss(x, token, t, loss, row_weight=weight, lse=lse, dlogits=dx, temperature=tau)
        L.distill_loss_backward(x, token, t, lse, weight, back, temperature=tau)
        scale = 1e30 / tau
        for got in (dx, back):
            # the logits themselves move a probability by 5 / tau
            assert float((got.double() / scale - want).abs().max()) <= (1.0 / 5001 + 0.125) * (64 * E + 3e-7 + 5 / tau)
