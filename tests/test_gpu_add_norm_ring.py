"""The norm's form for many rows, each variant of it against the FP64 definitions: rows side by side and one to a block, blocks of up to sixteen
warps, rows divided among two and four blocks, rows that start off 16 bytes, e4m3 with groups and with one scale a row, and their gradients.

The bounds are those of the other form (`test_gpu_add_norm.py`): a thread adds at most sixteen terms one behind the other, in pairs."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk
from paper_2609_19758_b200 import norm as N
from test_gpu_add_norm import E, TINY, grad_case, np64, rand, unit

pytestmark = pytest.mark.gpu

F32, F16, BF16, E4M3 = torch.float32, torch.float16, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


class Ring:
    """Asserts that the calls within are taken by the ring, all of them."""

    def __init__(self, calls):
        self.calls = calls

    def __enter__(self):
        self.before = fpsk.lib().fpsk_norm_ring_count()

    def __exit__(self, kind, value, trace):
        assert kind is not None or fpsk.lib().fpsk_norm_ring_count() - self.before == self.calls


# tokens, channels, elements between the rows: eight rows side by side to one row on four blocks; multiples of eight and odd
ALIGNED = [(700, 512, 0), (700, 64, 8), (300, 1024, 8), (200, 1536, 0), (150, 2048, 0), (90, 4096, 0), (90, 4104, 0), (80, 8192, 0), (80, 8200, 0),
           (60, 12288, 8), (40, 16384, 0), (40, 16640, 0), (40, 32768, 0)]
ODD = [(700, 513, 0), (301, 1021, 3), (300, 1501, 3), (300, 2051, 0), (150, 4097, 1), (151, 4101, 12), (90, 8191, 0), (80, 8201, 0), (60, 16383, 2),
       (40, 16385, 0), (40, 32767, 0)]
# enough rows that every block goes through its ring more than once
LONG, LONG_ODD = [(9500, 512, 0), (1500, 4096, 0), (600, 8192, 0), (520, 8200, 8), (320, 16384, 0), (160, 32768, 0)], \
    [(5301, 1021, 0), (3000, 1501, 1), (1501, 2051, 0), (800, 4101, 0), (520, 8201, 0), (160, 32767, 0)]
TYPES = [(F32, BF16, BF16), (BF16, F16, F32), (F16, F32, F16), (BF16, BF16, BF16), (F32, None, F32), (F32, F32, BF16)]
GRAD_TYPES = [(BF16, BF16), (F32, F32), (F16, F32), (F32, F16)]


@pytest.mark.parametrize("tokens,dim,pad,src,res,dst", [s + TYPES[(i + k) % 6] for i, s in enumerate(ALIGNED + ODD) for k in (0, 2, 3)]
                         + [s + TYPES[(i + k) % 6] for i, s in enumerate(LONG + LONG_ODD) for k in (0, 3)])
def test_forward(tokens, dim, pad, src, res, dst):
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = rand(g, tokens, dim, src, pad)
    residual = None if res is None else rand(g, tokens, dim, res, pad, 2.0)
    w = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    for w in (w.to(F16), None, w) if tokens * dim < 2e6 else (w,):
        y = torch.full((tokens, dim + pad), 7.0, dtype=dst, device="cuda")
        h = None if res is None else torch.full((tokens, dim + pad), 7.0, dtype=res, device="cuda")
        with Ring(1):
            N.add_rms_norm(x, residual, w, y[:, :dim], residual_out=None if h is None else h[:, :dim], eps=1e-5)
        h_ref, y_ref = D.add_norm(np64(x), None if residual is None else np64(residual), None if w is None else np64(w), 1e-5)
        assert np.all(np.abs(np64(y[:, :dim]) - y_ref) <= (unit(dst) + 64 * E) * np.abs(y_ref) + TINY[dst])
        assert bool((y[:, dim:] == 7.0).all())
        if h is not None:
            assert np.all(np.abs(np64(h[:, :dim]) - h_ref) <= (unit(res) + 2 * E) * np.abs(h_ref) + TINY[res])
            assert bool((h[:, dim:] == 7.0).all())
    if src == dst and res is not None:                                 # in place, both
        kept_y, kept_h = y[:, :dim].clone(), h[:, :dim].clone()
        with Ring(1):
            N.add_rms_norm(x, residual, w, x, residual_out=residual, eps=1e-5)
        assert torch.equal(x, kept_y) and torch.equal(residual, kept_h)


@pytest.mark.parametrize("tokens,dim,pad,group", [s + (group,) for s in ALIGNED for group in (0, 32, 64, 128, 256)] + [s + (group,) for s in LONG for group in (0, 128)])
def test_eight_bits(tokens, dim, pad, group):
    src, res = [(F32, BF16), (BF16, F32), (F16, None)][(dim + group // 32) % 3]
    g = torch.Generator(device="cuda").manual_seed(dim + group)
    x = rand(g, tokens, dim, src, pad)
    x[:, ::17] *= 30.0
    residual = None if res is None else rand(g, tokens, dim, res, pad)
    w = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    if group and dim > group:
        w[group:2 * group] = 0.0                                       # a group of zeros
    y = torch.full((tokens, dim + pad), 7.0, device="cuda").to(E4M3)
    groups = -(-dim // group) if group else 1
    scale = torch.full((tokens, groups + 1), 7.0, device="cuda")
    h = None if res is None else torch.empty(tokens, dim, dtype=res, device="cuda")
    with Ring(1):
        N.add_rms_norm(x, residual, w, y[:, :dim], residual_out=h, scale=scale[:, :groups], group=group, eps=1e-5)
    h_ref, y_ref = D.add_norm(np64(x), None if residual is None else np64(residual), np64(w), 1e-5)
    s_ref = D.e4m3_scales(y_ref, group)
    s = np64(scale)
    assert np.all(s[:, groups:] == 7.0) and bool((y[:, dim:].float() == 7.0).all())
    s = s[:, :groups]
    assert np.all(np.abs(s - s_ref) <= 66 * E * s_ref)
    want = y_ref / np.repeat(s_ref, group or dim, axis=1)[:, :dim]
    got = np64(y[:, :dim].float())
    assert np.all(np.abs(got - want) <= (2.0 ** -4 + 140 * E) * np.abs(want) + 2.0 ** -10)
    assert np.all(np.abs(got).max(1) == 448.0)
    if h is not None:
        assert np.all(np.abs(np64(h) - h_ref) <= (unit(res) + 2 * E) * np.abs(h_ref) + TINY[res])


def test_special_values():
    """Rows of zeros, NaN, infinities and very large values between ordinary ones, also where a row is divided among blocks."""
    for dim in (512, 4096, 8200, 16640):
        g = torch.Generator(device="cuda").manual_seed(dim)
        x = torch.randn(700 if dim < 4096 else 100, dim, generator=g, device="cuda")
        x[3] = 0.0
        x[10, dim - 1] = float("nan")
        x[20, 7] = float("inf")
        x[30] *= 1e15
        plain = torch.empty_like(x)
        with Ring(1):
            N.add_rms_norm(x, None, None, plain, eps=1e-30)
        fine = [r for r in range(x.shape[0]) if r not in (10, 20)]
        _, y_ref = D.add_norm(np64(x[fine]), None, None, 1e-30)
        assert np.all(np.abs(np64(plain[fine]) - y_ref) <= 65 * E * np.abs(y_ref))
        assert bool(torch.isnan(plain[10]).all()) and bool(torch.isnan(plain[20, 7])) and bool((plain[20, 8:] == 0).all())
        for group in (0, 128):
            groups = -(-dim // group) if group else 1
            q, scale = torch.empty_like(x).to(E4M3), torch.empty(x.shape[0], groups, device="cuda")
            with Ring(1):
                N.add_rms_norm(x, None, None, q, scale=scale, group=group, eps=1e-30)
            assert bool((scale[3] == 1).all()) and bool((q[3].float() == 0).all())
            assert bool(torch.isnan(scale[10]).all()) and bool(torch.isnan(q[10].float()).all()) and bool(torch.isnan(scale[20, 0]))
            assert np.all(np.abs(np64(scale[fine]) - D.e4m3_scales(y_ref, group)) <= 66 * E * D.e4m3_scales(y_ref, group))


def test_expanded_inputs_and_a_last_step_that_is_not_full():
    for tokens, dim in ((601, 512), (77, 2050), (75, 8201)):
        g = torch.Generator(device="cuda").manual_seed(dim)
        one, res = rand(g, 1, dim, F32), rand(g, tokens, dim, BF16)
        y, h, y1, h1 = (torch.empty(tokens, dim, dtype=BF16, device="cuda") for _ in range(4))
        with Ring(2):
            N.add_rms_norm(one.expand(tokens, dim), res, None, y, residual_out=h)
            N.add_rms_norm(one.repeat(tokens, 1), res, None, y1, residual_out=h1)
        assert torch.equal(y, y1) and torch.equal(h, h1)


@pytest.mark.parametrize("tokens,dim,pad,src,grad", [s + GRAD_TYPES[(i + k) % 4] for i, s in enumerate(ALIGNED + ODD) for k in (0, 1)]
                         + [s + GRAD_TYPES[i % 4] for i, s in enumerate(LONG + LONG_ODD)])
def test_backward(tokens, dim, pad, src, grad):
    g = torch.Generator(device="cuda").manual_seed(dim)
    h, dy, dh = grad_case(tokens, dim, src, grad, pad, g)
    ws = N.add_rms_norm_workspace(dim)
    w32 = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    for w, with_dh in ((w32, True), (None, True), (w32.to(BF16), False))[:3 if tokens * dim < 2e6 else 1]:
        dx = torch.full((tokens, dim + pad), 7.0, dtype=grad, device="cuda")
        dw = torch.full((dim,), 7.0, device="cuda")
        with Ring(1):
            N.add_rms_norm_backward(h, dy, w, dx[:, :dim], dw, ws, dh=dh if with_dh else None, eps=1e-5)
        dx_ref, mag, dw_ref, dw_mag = D.add_norm_grad(np64(h), None if w is None else np64(w), np64(dy), np64(dh) if with_dh else None, 1e-5)
        assert np.all(np.abs(np64(dx[:, :dim]) - dx_ref) <= unit(grad) * np.abs(dx_ref) + 256 * E * mag + TINY[grad])
        assert np.all(np.abs(np64(dw) - dw_ref) <= (tokens + 64) * E * dw_mag)
        assert bool((dx[:, dim:] == 7.0).all())
        only = torch.empty_like(dx)
        with Ring(1):
            N.add_rms_norm_backward(h, dy, w, only[:, :dim], dh=dh if with_dh else None, eps=1e-5)
        assert torch.equal(only[:, :dim], dx[:, :dim])
    for alias in ("dy", "dh"):                                         # in place
        a, b = torch.empty(tokens, dim + pad, dtype=grad, device="cuda")[:, :dim], torch.empty(tokens, dim + pad, dtype=grad, device="cuda")[:, :dim]
        a.copy_(dy)
        b.copy_(dh)
        want = torch.empty_like(dx)
        with Ring(2):
            N.add_rms_norm_backward(h, dy, w, want[:, :dim], dh=dh, eps=1e-5)
            N.add_rms_norm_backward(h, a, w, a if alias == "dy" else b, dh=b, eps=1e-5)
        assert torch.equal(a if alias == "dy" else b, want[:, :dim])
