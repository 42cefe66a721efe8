"""The decoder's operators at the edges that their own tests do not reach: the widest vocabulary, tensors whose offsets pass 32 bits, calls
at once on two streams, a first call inside a capture, tensors used in place by chained calls."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L
from paper_2609_19758_b200 import norm as N

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = 2.0 ** -24
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def test_the_widest_vocabulary():
    vocab = 1 << 23
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(1, vocab, generator=g, device="cuda")
    history = torch.tensor([[vocab - 1, 5, vocab - 1, 4000000]], dtype=torch.int32, device="cuda")
    x[0, vocab - 1] = 9.0
    token, lse = torch.empty(1, dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda")
    out = torch.empty(1, vocab, dtype=F16, device="cuda")
    L.adjust_logits(x, out, history=history, frequency=torch.full((1,), 0.5, device="cuda"), token=token, lse=lse)
    z, _ = D.adjust_logits(x[0].double().cpu().numpy(), history[0].tolist(), frequency=0.5)
    # z: one product and one difference (4 E of 10); lse: E of the exponents' size 15, powers 2 E, sums of vocab / 8 / 128 / 16 pieces one after another
    assert int(token) == int(z.argmax()) and abs(float(lse) - D.log_sum_exp(z)) <= 4 * E * 15 + (vocab / 8 / 128 / 16 + 64) * E
    assert np.all(np.abs(out[0].double().cpu().numpy() - z) <= 2.0 ** -11 * np.abs(z) + 40 * E + 2.0 ** -25)
    tok = torch.tensor([[vocab - 1, 0, 7000001]], device="cuda")
    t = torch.tensor([[1.0, 2.0, 0.5]], device="cuda")
    loss, dx = torch.empty(1, device="cuda"), torch.empty(1, vocab, device="cuda")
    L.distill_loss(x, tok, t, loss, dlogits=dx)
    l, d, _, mag, dmag = D.distill(x[0].double().cpu().numpy(), tok[0].tolist(), t[0].tolist(), 1.0, True)
    off = (vocab / 8 / 128 / 16 + 200) * E                             # the sum's, and 64 E and more of exponents up to 30
    assert abs(float(loss) - l) <= 64 * E * mag + off
    assert np.all(np.abs(dx[0].double().cpu().numpy() - d) <= 2 * off * dmag + 2.0 ** -126)
    with pytest.raises(RuntimeError):
        L.adjust_logits(torch.zeros(1, vocab + 1, dtype=F16, device="cuda"), token=token)


def test_offsets_beyond_32_bits():
    """The last rows of a call whose tensors have more than 2^31 elements are those of a call with them alone."""
    rows, vocab = 17000, 131072 + 8
    x = torch.empty(rows, vocab, dtype=BF16, device="cuda")
    x.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    assert x.numel() > 2 ** 31
    tok = torch.randint(0, vocab, (rows, 5), device="cuda", dtype=torch.int32)
    t = torch.randn(rows, 5, device="cuda")
    weight = torch.zeros(rows, device="cuda")
    weight[-3:] = 1.0                                                  # (the others are not read)
    loss, token = torch.empty(rows, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    one, pick = torch.empty(3, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    L.distill_loss(x, tok, t, loss, row_weight=weight)
    L.distill_loss(x[-3:], tok[-3:], t[-3:], one)
    # (other numbers of blocks to a row: other orders of the sums)
    assert float((loss[-3:] - one).abs().max()) <= (vocab / 1024 + 100) * E * 20
    L.adjust_logits(x, token=token)
    L.adjust_logits(x[-3:], token=pick)
    assert torch.equal(token[-3:], pick) and torch.equal(pick.long(), x[-3:].argmax(1))
    L.adjust_logits(x, x, mask=torch.full((1, -(-vocab // 32)), -2, dtype=torch.int32, device="cuda"),
                    mask_row=torch.where(torch.arange(rows, device="cuda") >= rows - 2, 0, -1).to(torch.int32))
    assert bool(torch.isneginf(x[-2:, ::32]).all()) and not bool(torch.isneginf(x[-2:, 1::32]).any()) and not bool(torch.isneginf(x[-3]).any())
    del x
    tokens, dim = 140000, 16384
    h = torch.empty(tokens, dim, dtype=BF16, device="cuda")
    h.normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    y, y1 = torch.empty_like(h), torch.empty(2, dim, dtype=BF16, device="cuda")
    N.add_rms_norm(h, None, None, y)
    N.add_rms_norm(h[-2:], None, None, y1)
    # (another form: the two are off by 64 E each before the rounding, a unit of BF16 apart at most)
    assert float((y[-2:].float() - y1.float()).abs().max()) <= 2.0 ** -8 * float(y1.float().abs().max())


def test_two_streams_at_once():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(300, 50304, generator=g, device="cuda")
    tok = torch.randint(0, 50304, (300, 40), generator=g, device="cuda", dtype=torch.int32)
    t = torch.randn(300, 40, generator=g, device="cuda")
    h = torch.randn(3000, 4096, generator=g, device="cuda").to(BF16)

    def call(stream):
        loss, dx = torch.empty(300, device="cuda"), torch.empty(300, 50304, dtype=BF16, device="cuda")
        y, s, dy, dw, ws = torch.empty_like(h), torch.empty_like(h), torch.empty_like(h), torch.empty(4096, device="cuda"), N.add_rms_norm_workspace(4096)
        token = torch.empty(300, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        return (loss, dx, y, dy, dw, token), lambda: (
            L.distill_loss(x, tok, t, loss, dlogits=dx, stream=stream), N.add_rms_norm(h, h, None, y, residual_out=s, stream=stream),
            N.add_rms_norm_backward(s, y, None, dy, dw, ws, dh=h, stream=stream), L.adjust_logits(x, token=token, history=tok, stream=stream))

    streams = [torch.cuda.Stream() for _ in range(3)]
    want, f = call(torch.cuda.current_stream())
    f()
    torch.cuda.synchronize()
    calls = [call(s) for s in streams]
    for _ in range(5):
        for _, f in calls:
            f()
    torch.cuda.synchronize()
    for got, _ in calls:
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_chained_in_place_calls():
    """Each launch overlaps the end of the one in front: a chain through the same buffers is what the calls give one by one."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(600, 2048, generator=g, device="cuda").to(BF16)
    w = 1 + 0.1 * torch.randn(2048, generator=g, device="cuda")

    def chain(sync):
        a, r = x.clone(), x.clone()
        for _ in range(40):
            N.add_rms_norm(a, r, w, a, residual_out=r)
            if sync:
                torch.cuda.synchronize()
        z = a.float()
        for i in range(20):
            L.adjust_logits(z, z, history=torch.full((600, 3), i, dtype=torch.int32, device="cuda"), frequency=torch.full((600,), 0.5, device="cuda"))
            if sync:
                torch.cuda.synchronize()
        return a, r, z

    assert all(torch.equal(a, b) for a, b in zip(chain(False), chain(True)))


def test_a_first_call_inside_a_capture():
    code = """
import torch
from paper_2609_19758_b200 import logits as L, norm as N
x = torch.randn(400, 4096, device="cuda")
tok, t = torch.randint(0, 4096, (400, 8), device="cuda", dtype=torch.int32), torch.randn(400, 8, device="cuda")
y, dx, dw, ws, ones = torch.empty_like(x), torch.empty_like(x), torch.empty(4096, device="cuda"), N.add_rms_norm_workspace(4096), torch.ones(4096, device="cuda")
loss, token, d = torch.empty(400, device="cuda"), torch.empty(400, dtype=torch.int32, device="cuda"), torch.empty_like(x)
def f():
    N.add_rms_norm(x, x, ones, y)
    N.add_rms_norm_backward(x, x, ones, dx, dw, ws, dh=x)
    L.distill_loss(x, tok, t, loss, dlogits=d)
    L.adjust_logits(x, token=token, history=tok)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    f()
graph.replay()
torch.cuda.synchronize()
first = [v.clone() for v in (y, dx, dw, loss, token, d)]
f()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, (y, dx, dw, loss, token, d)))
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
