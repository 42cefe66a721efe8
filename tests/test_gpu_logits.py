"""Penalties, biases and grammar masks on logits, the greedy token and the log-sum-exp, against the FP64 definitions.

Tolerances: E = 2^-24 is a rounding in FP32.  A logit meets one rounding for the repetition, one each for frequency c, + presence and the
subtraction, one for each of its biases: 4 E of the magnitudes that the oracle gives (biases counted there), and half a step of the
output's type."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E = 2.0 ** -24
TINY = {F32: 2.0 ** -149, F16: 2.0 ** -25, BF16: 2.0 ** -133}


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def cuda(a, dtype):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def np64(t):
    return t.double().cpu().numpy()


def pack(allowed):
    """(masks, vocab) booleans to words of 32 bits; the bits behind the vocabulary are set."""
    masks, vocab = allowed.shape
    words = -(-vocab // 32)
    bits = np.ones((masks, words * 32), dtype=np.uint32)
    bits[:, :vocab] = allowed
    packed = (bits.reshape(masks, words, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return torch.from_numpy(packed.view(np.int32)).cuda()


def make(r, rows, vocab, width, biases, masks, dtype, pad=0):
    """Inputs of a call, and the oracle's arguments for each of its rows."""
    x = torch.from_numpy(2.5 * r.normal(size=(rows, vocab + pad))).to(dtype).cuda()[:, :vocab]
    kw, per_row = {}, [{} for _ in range(rows)]
    if width:
        history = (vocab * r.random((rows, width)) ** 3).astype(np.int64).clip(max=vocab - 1)
        history[r.random((rows, width)) < 0.05] = -1
        history[r.random((rows, width)) < 0.05] = vocab                # no token either
        length = r.integers(0, width + 1, rows)
        length[0] = width
        prompt = r.integers(0, width + 1, rows)
        rep, freq, pres = (r.random(rows) * s + o for s, o in ((1.0, 0.6), (0.8, -0.2), (0.8, -0.2)))
        kw = dict(history=cuda(history, torch.int32), history_len=cuda(length, torch.int32), prompt_len=cuda(prompt, torch.int32),
                  repetition=cuda(rep, F32), frequency=cuda(freq, F32), presence=cuda(pres, F32))
        for i in range(rows):
            per_row[i] = dict(history=history[i, :length[i]], n_prompt=prompt[i], repetition=float(kw["repetition"][i]),
                              frequency=float(kw["frequency"][i]), presence=float(kw["presence"][i]))
    if biases:
        counts = r.integers(0, biases + 1, rows)
        ptr = np.concatenate([[0], np.cumsum(counts)])
        tokens = r.integers(-2, vocab + 2, ptr[-1])
        if ptr[-1] > 2:
            tokens[::3] = tokens[0]                                    # the same token again and again
        values = 3 * r.normal(size=ptr[-1])
        kw["bias"] = (cuda(ptr, torch.int32), cuda(tokens, torch.int32), cuda(values, F32))
        v32 = kw["bias"][2].double().cpu().numpy()
        for i in range(rows):
            per_row[i]["biases"] = list(zip(tokens[ptr[i]:ptr[i + 1]], v32[ptr[i]:ptr[i + 1]]))
    if masks:
        allowed = r.random((masks, vocab)) < r.choice([0.9, 3.0 / vocab], (masks, 1))
        which = r.integers(-1, masks, rows)
        kw["mask"], kw["mask_row"] = pack(allowed), cuda(which, torch.int32)
        for i in range(rows):
            per_row[i]["allowed"] = allowed[which[i]] if which[i] >= 0 else None
    return x, kw, per_row


def check(x, kw, per_row, out, token, lse):
    rows, vocab = x.shape
    raw = np64(x)
    for i in range(rows):
        z, mag = D.adjust_logits(raw[i], **per_row[i])
        tol = 4 * E * mag
        if out is not None:
            got = np64(out[i])
            u = torch.finfo(out.dtype).eps / 2
            fine = np.isfinite(z)
            assert np.array_equal(np.isneginf(got), np.isneginf(z))
            assert np.all(np.abs(got[fine] - z[fine]) <= (tol + u * np.abs(z) + TINY[out.dtype])[fine])
        if token is not None:
            t = int(token[i])
            if np.isneginf(z).all():
                assert t == -1 and float(lse[i]) == -np.inf
                continue
            assert z[t] + tol[t] >= (z - tol).max()
            # z log2(e) is rounded once and subtracted exactly; the powers and the sums (vocab / 512 of a lane behind one another, or fewer) as relative errors
            bound = tol.max() + 4 * E * np.abs(z[np.isfinite(z)]).max() + (vocab / 64 + 64) * E
            assert abs(float(lse[i]) - D.log_sum_exp(z)) <= bound


@pytest.mark.parametrize("rows,vocab,width,biases,masks,src,dst,pad", [
    (1, 1, 3, 2, 1, F32, F32, 0), (3, 31, 0, 0, 2, F32, F32, 0), (2, 33, 40, 5, 0, F16, F16, 0), (5, 1000, 300, 40, 3, F32, BF16, 3),
    (4, 4096, 17, 0, 0, BF16, F32, 0), (3, 4097, 0, 100, 2, BF16, BF16, 5), (7, 32000, 1000, 70, 4, F32, F32, 0), (2, 50257, 700, 16, 2, BF16, F32, 0),
    (1, 131072, 5000, 300, 1, F32, F16, 0), (150, 5003, 64, 3, 9, F16, F32, 1), (2, 270001, 100, 10, 2, F32, F32, 0), (1, 131072, 0, 0, 0, F32, F32, 0)])
def test_adjust(rows, vocab, width, biases, masks, src, dst, pad):
    r = np.random.default_rng(vocab)
    x, kw, per_row = make(r, rows, vocab, width, biases, masks, src, pad)
    before = x.clone()
    out = torch.full((rows, vocab + pad), 7.0, dtype=dst, device="cuda")
    token, lse = torch.full((rows,), 77, dtype=torch.int32, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    L.adjust_logits(x, out[:, :vocab], token=token, lse=lse, **kw)
    check(x, kw, per_row, out[:, :vocab], token, lse)
    assert bool((out[:, vocab:] == 7.0).all()) and torch.equal(x, before)
    # each output alone is the same
    only = torch.full_like(out, 7.0)
    L.adjust_logits(x, only[:, :vocab], **kw)
    assert torch.equal(only, out)
    t2, l2 = torch.empty_like(token), torch.empty_like(lse)
    L.adjust_logits(x, token=t2, **kw)
    L.adjust_logits(x, lse=l2, **kw)
    assert torch.equal(t2, token) and torch.equal(l2, lse)
    if src == dst:
        L.adjust_logits(x, x, **kw)                                    # in place
        assert torch.equal(x, out[:, :vocab])


def test_ties_infinities_and_nan():
    vocab = 9000
    x = torch.zeros(8, vocab, device="cuda")
    x[0, 5000] = x[0, 7000] = 3.0
    x[1] = -0.0
    x[1, 17] = 0.0                                                     # equal to -0: the first token
    x[2] = -float("inf")
    x[3] = -float("inf")
    x[3, 8999] = -1e30
    x[4, 4242] = float("nan")
    x[4, 4000] = float("inf")
    x[5, 100] = float("inf")
    x[6, 50] = float("nan")                                            # masked below
    x[6, 60] = 2.0
    x[7] = 1e38
    allowed = np.ones((1, vocab), dtype=bool)
    allowed[0, 50] = False
    which = cuda([-1, -1, -1, -1, -1, -1, 0, -1], torch.int32)
    out, token, lse = torch.empty_like(x), torch.empty(8, dtype=torch.int32, device="cuda"), torch.empty(8, device="cuda")
    L.adjust_logits(x, out, mask=pack(allowed), mask_row=which, token=token, lse=lse)
    assert token.tolist() == [5000, 0, -1, 8999, 4242, 100, 60, 0]
    l = lse.tolist()
    assert l[2] == -np.inf and l[3] == pytest.approx(-1e30, rel=4 * E) and np.isnan(l[4]) and l[5] == np.inf
    assert l[1] == pytest.approx(np.log(vocab), rel=64 * E) and l[6] == pytest.approx(np.log(vocab - 2 + np.exp(2.0)), rel=128 * E)
    assert l[7] == pytest.approx(1e38, rel=4 * E)
    assert float(out[6, 50]) == -np.inf and bool(torch.isnan(out[4, 4242]))


def test_masks_that_allow_nothing_or_are_missing():
    x = torch.randn(4, 100, device="cuda")
    allowed = np.zeros((2, 100), dtype=bool)
    allowed[1, 99] = True
    token, out = torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    L.adjust_logits(x, out, mask=pack(allowed), mask_row=cuda([0, 1, -1, -5], torch.int32), token=token, status=status)
    assert token[:2].tolist() == [-1, 99] and token[2:].tolist() == x[2:].argmax(1).tolist() and int(status) == 0
    assert torch.equal(out[2:], x[2:])
    L.adjust_logits(x, out, mask=pack(allowed), mask_row=cuda([0, 1, 2, -1], torch.int32), token=token, status=status)
    assert token[:3].tolist() == [-1, 99, -1] and int(status) == 10 and bool(torch.isneginf(out[2]).all())
    L.adjust_logits(x, mask=torch.empty(0, 4, dtype=torch.int32, device="cuda"), mask_row=cuda([-1] * 4, torch.int32), token=token)
    assert token.tolist() == x.argmax(1).tolist()


def test_biases_of_one_token_are_added_in_their_order():
    x = torch.zeros(1, 64, device="cuda")
    values = np.array([1e8, 3.0, -1e8, 0.25] * 20, dtype=np.float32)
    out = torch.empty_like(x)
    L.adjust_logits(x, out, bias=(cuda([0, 80], torch.int32), cuda([9] * 80, torch.int32), cuda(values, F32)))
    want = np.float32(0.0)
    for v in values:
        want = np.float32(want + v)
    assert float(out[0, 9]) == want and int((out != 0).sum()) <= 1


def test_many_of_the_same_token():
    """A count beyond 16 bits."""
    n = 70000
    x = torch.full((1, 50), 2.0, device="cuda")
    out = torch.empty_like(x)
    L.adjust_logits(x, out, history=torch.full((1, n), 7, dtype=torch.int32, device="cuda"), frequency=cuda([0.5], F32))
    assert float(out[0, 7]) == 2.0 - 0.5 * n and int((out == 2.0).sum()) == 49


def test_repeatable_captured_and_on_another_stream():
    r = np.random.default_rng(4)
    for rows, vocab in ((1, 131072), (40, 50257)):
        x, kw, _ = make(r, rows, vocab, 900, 33, 3, F32)

        def call(stream=None):
            o = torch.empty(rows, vocab, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
            return o, lambda: L.adjust_logits(x, o[0], token=o[1], lse=o[2], stream=stream, **kw)

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


def test_no_rows():
    x = torch.empty(0, 100, device="cuda")
    L.adjust_logits(x, torch.empty_like(x), token=torch.empty(0, dtype=torch.int32, device="cuda"))


def test_refusals():
    x, out = torch.zeros(3, 100, device="cuda"), torch.zeros(3, 100, device="cuda")
    token, three = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda")
    words = torch.zeros(3, 4, dtype=torch.int32, device="cuda")
    hist = torch.zeros(3, 5, dtype=torch.int32, device="cuda")
    ptr = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: L.adjust_logits(x), lambda: L.adjust_logits(x, out[:2]), lambda: L.adjust_logits(x, out.t()), lambda: L.adjust_logits(x[0], token=token),
                lambda: L.adjust_logits(x, out[:1].expand(3, 100)), lambda: L.adjust_logits(x, token=three), lambda: L.adjust_logits(x, token=token[:2]),
                lambda: L.adjust_logits(x, out, mask=words[:, :3]), lambda: L.adjust_logits(x, out, mask=words[:2]), lambda: L.adjust_logits(x, out, mask_row=token),
                lambda: L.adjust_logits(x, out, repetition=three), lambda: L.adjust_logits(x, out, history=hist[:2]), lambda: L.adjust_logits(x, out, history=hist, prompt_len=three),
                lambda: L.adjust_logits(x, out, history=hist, frequency=three.double()), lambda: L.adjust_logits(x, out, bias=(ptr[:3], token, three)),
                lambda: L.adjust_logits(x, out, bias=(ptr, token, three[:2])), lambda: L.adjust_logits(x.cpu(), out), lambda: L.adjust_logits(x, out.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: L.adjust_logits(x.double(), out), lambda: L.adjust_logits(x, "out"), lambda: L.adjust_logits(x, out, history=hist.long()),
                lambda: L.adjust_logits(x, out, mask=words.long())):
        with pytest.raises(TypeError):
            bad()
    assert bool((out == 0).all())
