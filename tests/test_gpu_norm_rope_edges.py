"""Norms and rotation at the edges of what the entry points take: eps = 0, kinds of heads without heads, gradients of gradients, and
gradients of an FP32 accumulator.  Tolerances as in test_gpu_norm_rope.py."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B

from test_gpu_norm_rope import E32, TINY, UNIT, _plain, close, projection, tables

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("tokens,hq,hk,dim,rot,inter,dtype", [
    (1, 4, 1, 128, 128, False, F32),         # most slots of a block are empty
    (7, 3, 2, 64, 32, True, BF16),
    (13, 28, 4, 96, 96, False, F16),         # heads that do not fill the slots, lanes behind the last channel
    (5, 2, 1, 256, 0, False, F32),
    (333, 40, 8, 80, 40, False, F32),        # several blocks, tokens that do not fill the last step
])
def test_backward_without_eps(tokens, hq, hk, dim, rot, inter, dtype):
    rng = np.random.default_rng(dim)
    q, k = projection(rng, tokens, (hq, hk), dim, dtype)
    gq, gk = projection(rng, tokens, (hq, hk), dim, BF16)
    cos, sin, c64, s64 = tables(50, rot)
    pos = torch.from_numpy(rng.integers(0, 50, tokens).astype(np.int32)).cuda()
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda()
    dq, dk = (torch.full((tokens, h, dim), 7.0, dtype=BF16, device="cuda") for h in (hq, hk))
    dw = [torch.full((dim,), 7.0, device="cuda") for _ in range(2)]
    A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, dq, dk, dw[0], dw[1], A.norm_rope_workspace(dim), w, w, eps=0.0, interleaved=inter)
    p = pos.cpu().numpy()
    for x, g, dx, dwt in ((q, gq, dq, dw[0]), (k, gk, dk, dw[1])):
        want, mag, want_w, mag_w = O.norm_rope_grad(x.double().cpu().numpy(), w.double().cpu().numpy(), g.double().cpu().numpy(), c64[p], s64[p],
                                                    rot, 0.0, inter)
        close(dx, want, UNIT[BF16] * np.abs(want) + 64 * E32 * mag)
        close(dwt, want_w, (256 + 32 + tokens * x.shape[1] / 8) * E32 * mag_w)


def test_many_tokens_backward_without_eps():
    """The form for large calls."""
    rng = np.random.default_rng(1)
    tokens, hq, hk, dim = 4000, 3, 2, 128
    q, k = projection(rng, tokens, (hq, hk), dim, F32)
    gq, gk = projection(rng, tokens, (hq, hk), dim, BF16)
    cos, sin, _, _ = tables(300, dim)
    pos = torch.from_numpy(rng.integers(0, 300, tokens).astype(np.int32)).cuda()
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda()
    dq, dk = (torch.empty(tokens, h, dim, dtype=BF16, device="cuda") for h in (hq, hk))
    dw = [torch.empty(dim, device="cuda") for _ in range(2)]
    A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, dq, dk, dw[0], dw[1], A.norm_rope_workspace(dim), w, w, eps=0.0)
    c, s = cos[pos.long()].double(), sin[pos.long()].double()
    for x, g, dwt in ((q, gq, dw[0]), (k, gk, dw[1])):
        u, um = _plain(g, None, c, -s, dim, False, 0.0)
        n = x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True))
        chain = tokens * x.shape[1] / (148 * 16) + 32 + 148 + 17 + 32
        assert bool(((dwt.double() - (u * n).sum((0, 1))).abs() <= chain * E32 * (um * n.abs()).sum((0, 1))).all())


@pytest.mark.parametrize("empty", ["q", "k"])
@pytest.mark.parametrize("tokens", [1, 40])
def test_a_kind_without_heads_has_a_weight_gradient_of_zero(empty, tokens):
    rng = np.random.default_rng(2)
    hq, hk = (0, 3) if empty == "q" else (3, 0)
    q, k = projection(rng, tokens, (hq, hk), 64, F32)
    gq, gk = projection(rng, tokens, (hq, hk), 64, BF16)
    cos, sin, c64, s64 = tables(50, 64)
    pos = torch.from_numpy(rng.integers(0, 50, tokens).astype(np.int32)).cuda()
    w = torch.ones(64, device="cuda")
    dq, dk = (torch.full((tokens, h, 64), 7.0, dtype=BF16, device="cuda") for h in (hq, hk))
    dw = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, dq, dk, dw[0], dw[1], A.norm_rope_workspace(64), w, w, eps=1e-5, status=status)
    assert int(status) == 0
    x, g, dx, there, none = (k, gk, dk, dw[1], dw[0]) if empty == "q" else (q, gq, dq, dw[0], dw[1])
    assert bool((none == 0).all())
    p = pos.cpu().numpy()
    want, mag, want_w, mag_w = O.norm_rope_grad(x.double().cpu().numpy(), np.ones(64), g.double().cpu().numpy(), c64[p], s64[p], 64, 1e-5)
    close(dx, want, UNIT[BF16] * np.abs(want) + 64 * E32 * mag)
    close(there, want_w, (256 + 32) * E32 * mag_w)


def test_a_second_derivative_is_refused():
    q, k = (torch.randn(3, 2, 32, device="cuda", requires_grad=True) for _ in range(2))
    w = torch.ones(32, device="cuda", requires_grad=True)
    cos, sin, _, _ = tables(10, 32)
    pos = torch.arange(3, dtype=torch.int32, device="cuda")
    qo, ko = A.QKNormRope.apply(q, k, w, w, cos, sin, pos, F32, 1e-5, False)
    dq, = torch.autograd.grad(qo.square().sum() + ko.sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (dq.square().sum() + q.square().sum()).backward()          # (the first term alone would be left out in silence)


@pytest.mark.parametrize("in_type,out_type", [(F32, BF16), (F32, F16), (BF16, F32), (F16, BF16), (BF16, BF16)])
def test_autograd_gradients_have_the_precision_of_the_inputs(in_type, out_type):
    """The gradient of an FP32 accumulator is not rounded to the type of the outputs on its way."""
    rng = np.random.default_rng(4)
    q, k = (t.contiguous().requires_grad_() for t in projection(rng, 9, (3, 2), 64, in_type))
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(64)).astype(np.float32)).cuda()
    cos, sin, c64, s64 = tables(50, 64)
    pos = torch.from_numpy(rng.integers(0, 50, 9).astype(np.int32)).cuda()
    gq, gk = projection(rng, 9, (3, 2), 64, out_type)
    qo, ko = A.QKNormRope.apply(q, k, w, w, cos, sin, pos, out_type, 1e-5, False)
    assert qo.dtype == ko.dtype == out_type
    torch.autograd.backward((qo, ko), (gq, gk))
    p = pos.cpu().numpy()
    for x, g in ((q, gq), (k, gk)):
        assert x.grad.dtype == in_type
        want, mag, _, _ = O.norm_rope_grad(x.detach().double().cpu().numpy(), w.double().cpu().numpy(), g.double().cpu().numpy(), c64[p], s64[p], 64, 1e-5)
        close(x.grad, want, UNIT[in_type] * np.abs(want) + TINY[in_type] + 64 * E32 * mag)
