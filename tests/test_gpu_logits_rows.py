"""Adjusted logits where the kernel goes on from row to row, and in place with the token and the log-sum-exp."""
import numpy as np
import pytest
import torch

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import logits as L
from test_gpu_logits import check, make

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("rows,vocab,width,biases,masks,src,dst", [
    (2000, 3001, 64, 5, 9, F32, F32), (900, 20000, 100, 20, 0, BF16, F32), (1000, 3002, 9000, 4, 3, F16, F16), (1300, 3000, 0, 0, 5, F32, BF16),
    (700, 50257, 30, 3, 4, BF16, BF16), (1500, 5000, 0, 30, 0, F16, F32)])
def test_many_rows_of_a_cluster(rows, vocab, width, biases, masks, src, dst):
    """More rows than clusters fit the device, so that words, keys, rings and barriers are used for one row after another."""
    x, kw, per_row = make(np.random.default_rng(vocab), rows, vocab, width, biases, masks, src)
    out, token, lse = torch.empty(rows, vocab, dtype=dst, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    L.adjust_logits(x, out, token=token, lse=lse, **kw)
    check(x, kw, per_row, out, token, lse)
    only = torch.empty_like(out)
    L.adjust_logits(x, only, **kw)
    assert torch.equal(only, out)
    if src == dst:
        y = x.clone()
        L.adjust_logits(y, y, **kw)
        assert torch.equal(y, out)


@pytest.mark.parametrize("rows,vocab,width,biases,masks,src,pad", [
    (1, 1, 3, 2, 1, F32, 0), (5, 4097, 300, 400, 3, F32, 3), (4, 32000, 1000, 70, 2, BF16, 0), (3, 50257, 10, 0, 2, F16, 1), (700, 3001, 64, 5, 9, F32, 0),
    (2, 131072, 0, 300, 1, F32, 0), (6, 9999, 0, 0, 2, BF16, 5)])
def test_in_place_with_the_token_and_the_log_sum_exp(rows, vocab, width, biases, masks, src, pad):
    """The usual call of a server: the rows are read through the ring and written where they stand."""
    x, kw, per_row = make(np.random.default_rng(vocab + 1), rows, vocab, width, biases, masks, src, pad)
    out, token, lse = torch.empty(rows, vocab, dtype=src, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    L.adjust_logits(x, out, token=token, lse=lse, **kw)
    check(x, kw, per_row, out, token, lse)
    for want in (dict(token=True, lse=True), dict(token=True), dict(lse=True)):
        whole = torch.full((rows, vocab + pad), 7.0, dtype=src, device="cuda")
        y = whole[:, :vocab]
        y.copy_(x)
        t2, l2 = torch.full_like(token, 77), torch.full_like(lse, 7.0)
        L.adjust_logits(y, y, token=t2 if "token" in want else None, lse=l2 if "lse" in want else None, **kw)
        assert torch.equal(y, out) and bool((whole[:, vocab:] == 7.0).all())
        assert "token" not in want or torch.equal(t2, token)
        assert "lse" not in want or torch.equal(l2, lse)


def test_a_long_list_that_names_one_token_again_and_again():
    """Entries behind a token's first one are done with as soon as they have met it: a list of n entries of one token takes n steps of one thread, not
    n for each entry (the other blocks of the row wait, and give up after a second)."""
    n, vocab = 200000, 40000
    r = np.random.default_rng(0)
    values = r.integers(-8, 9, n).astype(np.float32)                   # (sums that FP32 holds)
    tokens = np.full(n, 777, dtype=np.int64)
    tokens[::1000] = np.arange(200) * 150
    x = torch.zeros(2, vocab, device="cuda")
    out, token, status = torch.empty_like(x), torch.empty(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    bias = tuple(torch.tensor(a, dtype=t, device="cuda") for a, t in ((np.array([0, n, n]), torch.int32), (tokens, torch.int32), (values, F32)))
    L.adjust_logits(x, out, bias=bias, token=token, status=status)
    want = np.zeros(vocab)
    np.add.at(want, tokens, values.astype(np.float64))
    assert int(status) == 0 and np.array_equal(out[0].double().cpu().numpy(), want) and bool((out[1] == 0).all())
    assert token.tolist() == [int(want.argmax()), 0]
