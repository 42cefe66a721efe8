"""Residual addition and RMS norm, forward and backward, against the FP64 definitions.

Tolerances: E = 2^-24 is a rounding in FP32, u half a step of the output type.  A sum of squares adds at most dim / 32 terms on a lane one
behind the other (8 to 32 in practice: a row has up to 1024 lanes) and ten or more of the lanes' sums, each off by E at most, relative; r takes half of that
and two units of its own, the products three more: 64 E covers all of y's error but its own rounding."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import norm as N

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn
E = 2.0 ** -24
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -24, BF16: 2.0 ** -133}


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def unit(t):
    return torch.finfo(t).eps / 2


def rand(g, tokens, dim, dtype, pad=0, scale=1.0):
    """Rows of a wider tensor where pad > 0."""
    return (scale * torch.randn(tokens, dim + pad, generator=g, device="cuda")).to(dtype)[:, :dim]


def np64(t):
    return t.double().cpu().numpy()


CASES = [(1, 4096, F32, BF16, BF16, 0), (3, 1, F32, None, F32, 0), (2, 7, F16, F16, F16, 0), (5, 8, BF16, F32, BF16, 0), (9, 100, F32, F16, F16, 4),
         (300, 256, BF16, BF16, F32, 0), (33, 513, F32, None, BF16, 1), (17, 1024, F16, F32, F16, 8), (4, 2050, F32, F32, F32, 0),
         (601, 2048, F32, BF16, BF16, 0), (7, 4100, BF16, BF16, BF16, 12), (3, 8200, F32, F16, F16, 0), (2, 16385, F32, BF16, BF16, 0),
         (2, 32768, F32, F32, BF16, 0), (2, 32767, BF16, None, F16, 0)]


@pytest.mark.parametrize("tokens,dim,src,res,dst,pad", CASES)
def test_forward(tokens, dim, src, res, dst, pad):
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = rand(g, tokens, dim, src, pad)
    residual = None if res is None else rand(g, tokens, dim, res, pad, 2.0)
    for w in (None, 1 + 0.3 * torch.randn(dim, generator=g, device="cuda"), (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(BF16)):
        y = torch.full((tokens, dim + pad), 7.0, dtype=dst, device="cuda")
        h = None if res is None else torch.full((tokens, dim + pad), 7.0, dtype=res, device="cuda")
        N.add_rms_norm(x, residual, w, y[:, :dim], residual_out=None if h is None else h[:, :dim], eps=1e-5)
        h_ref, y_ref = D.add_norm(np64(x), None if residual is None else np64(residual), None if w is None else np64(w), 1e-5)
        assert np.all(np.abs(np64(y[:, :dim]) - y_ref) <= (unit(dst) + 64 * E) * np.abs(y_ref) + TINY[dst])
        if h is not None:
            assert np.all(np.abs(np64(h[:, :dim]) - h_ref) <= (unit(res) + 2 * E) * np.abs(h_ref) + TINY[res])
            assert bool((h[:, dim:] == 7.0).all())
        assert bool((y[:, dim:] == 7.0).all())                         # what lies between the rows is left alone


@pytest.mark.parametrize("tokens,dim,src,res,group,pad", [(5, 4096, F32, BF16, 128, 0), (3, 4096, F32, F32, 0, 0), (7, 100, F16, F16, 32, 4), (2, 33, F32, None, 32, 0),
                                                          (4, 2050, BF16, BF16, 256, 0), (257, 512, F32, F16, 64, 0), (2, 16392, F32, BF16, 0, 8), (3, 8, F32, None, 0, 0),
                                                          (2, 32768, F32, BF16, 256, 0)])
def test_eight_bits(tokens, dim, src, res, group, pad):
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = rand(g, tokens, dim, src, pad)
    x[:, ::17] *= 30.0
    residual = None if res is None else rand(g, tokens, dim, res, pad)
    w = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    if group and dim > group:
        w[group:2 * group] = 0.0                                       # a group of zeros
    y = torch.zeros(tokens, dim + pad, dtype=F32, device="cuda").to(E4M3)
    groups = -(-dim // group) if group else 1
    scale = torch.full((tokens, groups + 1), 7.0, device="cuda")
    N.add_rms_norm(x, residual, w, y[:, :dim], scale=scale[:, :groups], group=group, eps=1e-5)
    _, y_ref = D.add_norm(np64(x), None if residual is None else np64(residual), np64(w), 1e-5)
    s_ref = D.e4m3_scales(y_ref, group)
    s = np64(scale)
    assert np.all(s[:, groups:] == 7.0)
    s = s[:, :groups]
    assert np.all(np.abs(s - s_ref) <= 66 * E * s_ref)
    want = y_ref / np.repeat(s_ref, group or dim, axis=1)[:, :dim]
    got = np64(y[:, :dim].float())
    # half a step of e4m3 (2^-4 relative, 2^-10 among the subnormals), of a quotient off by 132 E
    assert np.all(np.abs(got - want) <= (2.0 ** -4 + 140 * E) * np.abs(want) + 2.0 ** -10)
    assert np.abs(got).max() == 448.0


def test_in_place():
    g = torch.Generator(device="cuda").manual_seed(3)
    for dim in (512, 2050, 16384):
        x, residual, w = rand(g, 9, dim, BF16), rand(g, 9, dim, BF16), torch.rand(dim, generator=g, device="cuda")
        y, h = torch.empty_like(x), torch.empty_like(x)
        N.add_rms_norm(x, residual, w, y, residual_out=h)
        x2, r2 = x.clone(), residual.clone()
        N.add_rms_norm(x2, r2, w, x2, residual_out=r2)
        assert torch.equal(x2, y) and torch.equal(r2, h)
        dy, dh = rand(g, 9, dim, BF16), rand(g, 9, dim, BF16)
        dx = torch.empty_like(x)
        N.add_rms_norm_backward(h, dy, w, dx, dh=dh)
        for alias in ("dy", "dh"):
            a, b = dy.clone(), dh.clone()
            N.add_rms_norm_backward(h, a, w, a if alias == "dy" else b, dh=b)
            assert torch.equal(a if alias == "dy" else b, dx)


def test_special_values():
    """Rows of zeros, of infinities and NaN, of very large and very small values; each row is by itself."""
    dim = 1000
    x = torch.ones(6, dim, device="cuda")
    x[0] = 0.0
    x[1, 5] = float("nan")
    x[2, 7] = float("inf")
    x[3] *= 1e15
    x[4] *= 1e-12
    y = torch.empty(6, dim, device="cuda")
    N.add_rms_norm(x, None, None, y, eps=1e-30)
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1]).all())
    assert bool(torch.isnan(y[2, 7])) and bool((y[2, :7] == 0).all())
    assert bool((y[3:] - 1).abs().max() <= 64 * E)
    q, scale = torch.empty(6, dim, device="cuda").to(E4M3), torch.empty(6, 8, device="cuda")
    N.add_rms_norm(x, None, None, q, scale=scale, group=128, eps=1e-30)
    assert bool((scale[0] == 1).all()) and bool((q[0].float() == 0).all())
    assert bool(torch.isnan(scale[1]).all()) and bool(torch.isnan(q[1].float()).all())
    assert bool(torch.isnan(scale[2, 0])) and bool((scale[2, 1:] == 1).all()) and bool((q[2].float()[128:] == 0).all())
    assert bool((q[3:].float() == 448).all())
    row = torch.empty(6, 1, device="cuda")
    N.add_rms_norm(x, None, None, q, scale=row, eps=1e-30)
    assert bool(torch.isnan(row[1:3]).all()) and bool((row[0] == 1).all()) and bool(torch.isnan(q[1].float()).all())
    # a norm of zeros and eps = 0 is 0 times infinity
    N.add_rms_norm(x[:1], None, None, y[:1], eps=0.0)
    assert bool(torch.isnan(y[0]).all())


def grad_case(tokens, dim, src, grad, pad, g):
    h = rand(g, tokens, dim, src, pad, 1.5)
    dy, dh = rand(g, tokens, dim, grad, pad), rand(g, tokens, dim, grad, pad)
    return h, dy, dh


@pytest.mark.parametrize("tokens,dim,src,grad,pad", [(1, 4096, BF16, BF16, 0), (3, 1, F32, F32, 0), (2, 7, F16, F16, 0), (700, 64, BF16, BF16, 0), (40, 513, F32, F16, 1),
                                                     (37, 2050, F16, F32, 0), (310, 2048, F32, F32, 0), (5, 4100, BF16, BF16, 12), (4, 8200, F16, F16, 0),
                                                     (3, 16385, F32, BF16, 0), (2, 32768, BF16, F32, 0), (900, 1000, F32, BF16, 0), (1500, 8, F32, F32, 0)])
def test_backward(tokens, dim, src, grad, pad):
    g = torch.Generator(device="cuda").manual_seed(dim)
    h, dy, dh = grad_case(tokens, dim, src, grad, pad, g)
    ws = N.add_rms_norm_workspace(dim)
    for w, with_dh in ((1 + 0.3 * torch.randn(dim, generator=g, device="cuda"), True), (None, True), ((1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(F16), False)):
        dx = torch.full((tokens, dim + pad), 7.0, dtype=grad, device="cuda")
        dw = torch.full((dim,), 7.0, device="cuda")
        N.add_rms_norm_backward(h, dy, w, dx[:, :dim], dw, ws, dh=dh if with_dh else None, eps=1e-5)
        dx_ref, mag, dw_ref, dw_mag = D.add_norm_grad(np64(h), None if w is None else np64(w), np64(dy), np64(dh) if with_dh else None, 1e-5)
        # r and the mean are off by 64 E each, r enters three times
        assert np.all(np.abs(np64(dx[:, :dim]) - dx_ref) <= unit(grad) * np.abs(dx_ref) + 256 * E * mag + TINY[grad])
        # a column adds one product a token, in whatever order: at most `tokens` additions, and what r is off by
        assert np.all(np.abs(np64(dw) - dw_ref) <= (tokens + 64) * E * dw_mag)
        assert bool((dx[:, dim:] == 7.0).all())
        only = torch.empty_like(dx)
        N.add_rms_norm_backward(h, dy, w, only[:, :dim], dh=dh if with_dh else None, eps=1e-5)           # a weight that is not trained
        assert torch.equal(only[:, :dim], dx[:, :dim])


def test_no_tokens():
    for dim in (8, 4096):
        e = torch.empty(0, dim, device="cuda")
        N.add_rms_norm(e, e, None, torch.empty_like(e), residual_out=torch.empty_like(e))
        dw = torch.full((dim,), 7.0, device="cuda")
        N.add_rms_norm_backward(e, e, None, torch.empty_like(e), dw, N.add_rms_norm_workspace(dim))
        assert bool((dw == 0).all())


def test_rows_that_are_one_row():
    """Inputs may be expanded, outputs not."""
    x = torch.randn(1, 256, device="cuda")
    y, y1 = torch.empty(5, 256, device="cuda"), torch.empty(1, 256, device="cuda")
    N.add_rms_norm(x.expand(5, 256), x.expand(5, 256), None, y)
    N.add_rms_norm(x, x, None, y1)
    assert torch.equal(y, y1.expand(5, 256))
    with pytest.raises(ValueError, match="share"):
        N.add_rms_norm(y, None, None, y1.expand(5, 256))


@pytest.mark.parametrize("tokens,dim", [(3, 2050), (700, 4096)])
def test_repeatable_captured_and_on_another_stream(tokens, dim):
    g = torch.Generator(device="cuda").manual_seed(1)
    h, dy, dh = grad_case(tokens, dim, BF16, BF16, 0, g)
    w = torch.rand(dim, generator=g, device="cuda")

    def call(stream=None):
        y, s, dx, dw, ws = torch.empty_like(h), torch.empty_like(h), torch.empty_like(h), torch.empty(dim, device="cuda"), N.add_rms_norm_workspace(dim)
        return (y, s, dx, dw), lambda: (N.add_rms_norm(h, dh, w, y, residual_out=s, stream=stream), N.add_rms_norm_backward(h, dy, w, dx, dw, ws, dh=dh, stream=stream))

    first, f = call()
    f()
    torch.cuda.synchronize()
    again, f = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    kept = h.clone()
    h.mul_(2.0)
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(first[0], again[0])
    h.copy_(kept)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    third, f = call(st)
    torch.cuda.synchronize()
    f()
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, third))


@pytest.mark.parametrize("src,res,dst,wtype", [(F32, BF16, BF16, F32), (BF16, BF16, BF16, BF16), (F32, None, F32, F32), (F16, F32, F16, F32)])
def test_autograd(src, res, dst, wtype):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = rand(g, 11, 300, src).requires_grad_()
    residual = None if res is None else rand(g, 11, 300, res).requires_grad_()
    w = (1 + 0.3 * torch.randn(300, generator=g, device="cuda")).to(wtype).requires_grad_()
    y, h = N.AddRMSNorm.apply(x, residual, w, dst, 1e-5)
    gy, gh = rand(g, 11, 300, dst), rand(g, 11, 300, h.dtype)
    torch.autograd.backward([y, h], [gy, gh])
    dx_ref, mag, dw_ref, dw_mag = D.add_norm_grad(np64(h.detach()), np64(w.detach()), np64(gy), np64(gh), 1e-5)
    for t in (x, residual):
        if t is not None:
            assert t.grad.dtype == t.dtype
            assert np.all(np.abs(np64(t.grad) - dx_ref) <= 2 * unit(t.dtype) * np.abs(dx_ref) + 256 * E * mag + TINY[t.dtype])
    assert np.all(np.abs(np64(w.grad) - dw_ref) <= unit(wtype) * np.abs(dw_ref) + 128 * E * dw_mag)
    # one of the outputs unused
    x.grad = None
    y, _ = N.AddRMSNorm.apply(x, residual, w, dst, 1e-5)
    y.backward(gy)
    dx_ref, mag, _, _ = D.add_norm_grad(np64(h.detach()), np64(w.detach()), np64(gy), None, 1e-5)
    assert np.all(np.abs(np64(x.grad) - dx_ref) <= 2 * unit(src) * np.abs(dx_ref) + 256 * E * mag + TINY[src])


def test_refusals():
    x, y, w = torch.zeros(3, 64, device="cuda"), torch.zeros(3, 64, device="cuda"), torch.zeros(64, device="cuda")
    q, s = y.to(E4M3), torch.zeros(3, 1, device="cuda")
    for bad in (lambda: N.add_rms_norm(x, x[:2], w, y), lambda: N.add_rms_norm(x, None, w[:32], y), lambda: N.add_rms_norm(x, None, w, y.t()),
                lambda: N.add_rms_norm(x[0], None, w, y[0]), lambda: N.add_rms_norm(x.cpu(), None, w, y), lambda: N.add_rms_norm(x, None, w, y.cpu()),
                lambda: N.add_rms_norm(x, x, w, y, residual_out=y.half()), lambda: N.add_rms_norm(x, None, w, q, scale=s.expand(3, 2)),
                lambda: N.add_rms_norm(x, None, w, y, scale=s), lambda: N.add_rms_norm(x, None, w, q, scale=s, group=32),
                lambda: N.add_rms_norm_backward(x, y, w, y.half()), lambda: N.add_rms_norm_backward(x, y, w, y, w.half(), torch.zeros(1 << 20, device="cuda")),
                lambda: N.add_rms_norm_backward(x, y, w, y.clone(), dh=y.half())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: N.add_rms_norm("x", None, w, y), lambda: N.add_rms_norm(x.double(), None, w, y), lambda: N.add_rms_norm(x, None, w, q),
                lambda: N.add_rms_norm(x, None, w, y, eps="1"), lambda: N.add_rms_norm(x, None, w, q, scale=s.half())):
        with pytest.raises(TypeError):
            bad()
    wide = torch.zeros(1, 32769, device="cuda")
    for bad in (lambda: N.add_rms_norm(x, None, w, y, eps=-1.0), lambda: N.add_rms_norm(x, None, w, y, eps=float("nan")),
                lambda: N.add_rms_norm(x, None, w, y, group=32), lambda: N.add_rms_norm(x, None, w, q, scale=torch.zeros(3, 4, device="cuda"), group=16),
                lambda: N.add_rms_norm(wide, None, None, wide.clone()), lambda: N.add_rms_norm_workspace(0), lambda: N.add_rms_norm_workspace(32769),
                lambda: N.add_rms_norm_backward(x, y, w, y.clone(), w.clone()),
                lambda: N.add_rms_norm_backward(x, y, w, y.clone(), w.clone(), torch.zeros(256, device="cuda"))):
        with pytest.raises(RuntimeError):
            bad()
