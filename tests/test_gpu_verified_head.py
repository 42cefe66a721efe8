"""The verified head over many steps: its workspaces do not grow with the lengths of the batches, and serve all of its products."""
import pytest
import torch

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import decoder as M
from paper_2609_19758_b200 import fpsk

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def test_workspaces_do_not_grow_with_the_batches_lengths():
    g = torch.Generator(device="cuda").manual_seed(0)
    head = M.VerifiedHead((torch.randn(256, 1000, generator=g, device="cuda") / 16).half())
    before = torch.cuda.memory_allocated()
    lengths = list(range(8, 600, 8))
    for rows in lengths + lengths[::-1]:
        x = torch.randn(rows, 256, generator=g, device="cuda").half()
        token = torch.randint(0, 1000, (rows, 4), generator=g, device="cuda", dtype=torch.int32)
        head.distill(x, token, torch.zeros(rows, 4, device="cuda"))
        head.next_tokens(x)
        assert not head.fired()
    need = max(int(fpsk.lib().fpsk_probe_workspace_bytes(1, k, n)) for k, n in [(256, 1000), (1000, 256)] + [(rows, 256) for rows in lengths])
    del x, token
    held = torch.cuda.memory_allocated() - before
    assert held <= 4 * need, (held, need)                              # (the last is below twice what is needed, all below twice the last)
    # a fault is seen in a product of each shape
    for a, b in ((torch.randn(40, 256, device="cuda").half(), head.weight), (torch.randn(1000, 592, device="cuda").half(), torch.randn(592, 256, device="cuda").half())):
        head.product(a, b, fault=(3, 5, 1e4))
        assert head.fired()
        head.product(a, b)
        assert not head.fired()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 2, 7])
def test_few_rows_and_rows_without_weight(rows, dtype):
    """A training step of one position, whose logits' gradient is a single column when it is transposed, and one without any weight."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    head = M.VerifiedHead((torch.randn(256, 3000, generator=g, device="cuda") / 16).to(dtype))
    x = torch.randn(rows, 256, generator=g, device="cuda").to(dtype)
    token = torch.randint(0, 3000, (rows, 5), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randn(rows, 5, generator=g, device="cuda")
    loss, dx, dw = head.distill(x, token, t)
    assert not head.fired() and dx.shape == x.shape and dw.shape == head.weight.shape
    xd, wd = x.double().requires_grad_(), head.weight.double().requires_grad_()
    logq, logp = torch.log_softmax(xd @ wd, -1), torch.log_softmax(t.double(), -1)
    want = (logp.exp() * (logp - logq.gather(1, token.long()))).sum(-1)
    want.sum().backward()
    # as in the decoder's own test: the logits' gradient is rounded to 16 bits, the products are FP32
    u = torch.finfo(dtype).eps / 2
    assert float((loss.double() - want.detach()).abs().max()) <= 2.0 ** -16 * float(want.detach().abs().max())
    for got, ref in ((dx, xd.grad), (dw, wd.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2 * u + 2.0 ** -16
    loss, dx, dw = head.distill(x, token, t, torch.zeros(rows, device="cuda"))
    assert not head.fired() and not bool(loss.any()) and not bool(dx.any()) and not bool(dw.any())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,weight", [(160, 3000, 1.0 / 4096), (64, 40000, 1.0 / 65536), (3, 3000, 1e-3), (1, 3000, 1e-3), (2, 3000, 1e-12), (40, 3000, 3e4)])
def test_weights_of_any_size(rows, vocab, weight, dtype):
    """Gradients of a mean over many positions (or of a scaled loss): the logits' gradient is rounded relative to itself, not to what FP16 can
    hold.  Bounds as for weights of 1."""
    g = torch.Generator(device="cuda").manual_seed(vocab + rows)
    head = M.VerifiedHead((torch.randn(256, vocab, generator=g, device="cuda") / 16).to(dtype))
    x = torch.randn(rows, 256, generator=g, device="cuda").to(dtype)
    token = torch.randint(0, vocab, (rows, 6), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randn(rows, 6, generator=g, device="cuda")
    w = weight * (0.5 + torch.rand(rows, generator=g, device="cuda"))
    if rows > 8:
        w[::5] = 0.0
    loss, dx, dw = head.distill(x, token, t, w, temperature=1.5)
    assert not head.fired()
    xd, wd = x.double().requires_grad_(), head.weight.double().requires_grad_()
    logq, logp = torch.log_softmax(xd @ wd / 1.5, -1), torch.log_softmax(t.double() / 1.5, -1)
    want = (logp.exp() * (logp - logq.gather(1, token.long()))).sum(-1)
    (want * w.double()).sum().backward()
    u = torch.finfo(dtype).eps / 2
    live = w != 0
    assert float((loss.double() - want.detach())[live].abs().max()) <= 2.0 ** -16 * float(want.detach().abs().max())
    for got, ref in ((dx, xd.grad), (dw, wd.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2 * u + 2.0 ** -16


@pytest.mark.parametrize("vocab", [131080, 151936, 200001, 300000])
def test_wide_vocabularies(vocab):
    """More columns, or channels to sum over, than one probe takes: the product is probed in parts, and a fault is seen in each."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    rows, hidden = 24, 64
    head = M.VerifiedHead((torch.randn(hidden, vocab, generator=g, device="cuda") / 8).half())
    x = torch.randn(rows, hidden, generator=g, device="cuda").half()
    picked = head.next_tokens(x)
    assert not head.fired()
    z = x.double() @ head.weight.double()
    # (products of FP16 are exact in FP32, sums of 64 of them off by 64 roundings of at most 64 x 4 x 4 / 8)
    assert float((z.amax(1) - z.gather(1, picked.long()[:, None])[:, 0]).abs().max()) <= 2 * 64 * 2.0 ** -24 * 128
    for column in (0, vocab // 2, vocab - 1):
        head.next_tokens(x, fault=(5, column, 30.0))
        assert head.fired()
    token = torch.randint(0, vocab, (rows, 6), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randn(rows, 6, generator=g, device="cuda")
    loss, dx, dw = head.distill(x, token, t)
    assert not head.fired()
    xd, wd = x.double().requires_grad_(), head.weight.double().requires_grad_()
    logq, logp = torch.log_softmax(xd @ wd, -1), torch.log_softmax(t.double(), -1)
    (logp.exp() * (logp - logq.gather(1, token.long()))).sum().backward()
    for got, ref in ((dx, xd.grad), (dw, wd.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -10 + 2.0 ** -16
    a = torch.randn(40, vocab, generator=g, device="cuda").half()
    for _ in range(2):
        head.product(a, head.weight.t().contiguous(), fault=(3, 5, 3e4))
        assert head.fired()
        assert head.product(a, head.weight.t().contiguous()).shape == (40, hidden) and not head.fired()
