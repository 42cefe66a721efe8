"""The FP64 definitions of the decoder's operators against differences and against cases that can be worked out by hand."""
import numpy as np
import pytest

from oracle import decoder_oracle as D


@pytest.mark.parametrize("eps", [0.0, 1e-6, 0.3])
def test_norm_gradients_against_differences(eps):
    r = np.random.default_rng(1)
    h, w, dy, dh = (r.normal(size=s) for s in ((3, 7), (7,), (3, 7), (3, 7)))
    dx, _, dw, _ = D.add_norm_grad(h, w, dy, dh, eps)

    def f(h, w):
        return (dy * D.add_norm(h, None, w, eps)[1]).sum() + (dh * h).sum()

    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = 1e-6
        assert (f(h + e, w) - f(h - e, w)) / 2e-6 == pytest.approx(dx[i], abs=1e-7, rel=1e-6)
    for i in range(7):
        e = np.zeros(7)
        e[i] = 1e-6
        assert (f(h, w + e) - f(h, w - e)) / 2e-6 == pytest.approx(dw[i], abs=1e-7, rel=1e-6)


def test_norm_by_hand():
    h, y = D.add_norm([[3.0, 0.0]], [[0.0, 4.0]], np.array([1.0, 2.0]), 0.0)
    assert h.tolist() == [[3.0, 4.0]] and np.allclose(y, [[3.0 / 12.5 ** 0.5, 8.0 / 12.5 ** 0.5]])
    s = D.e4m3_scales(np.array([[0.0, 0.0, 1.0, -896.0, 448.0]]), 2)
    assert s.tolist() == [[1.0, 2.0, 1.0]]


def test_logits_by_hand():
    z, _ = D.adjust_logits([2.0, -2.0, 1.0, 5.0, 0.0], [0, 1, 0, 0, -1, 9], 1, 2.0, 0.25, 0.5, [(2, 1.0), (2, 0.5), (7, 3.0)], [True, True, True, False, True])
    assert z.tolist() == [1.0 - 0.5 - 0.5, -4.0 - 0.25 - 0.5, 2.5, -np.inf, 0.0]
    assert D.log_sum_exp(np.full(4, -np.inf)) == -np.inf
    assert D.log_sum_exp(np.zeros(4)) == pytest.approx(np.log(4))


@pytest.mark.parametrize("normalize,temperature", [(True, 1.0), (True, 2.5), (False, 1.0), (False, 0.5)])
def test_distillation_gradients_against_differences(normalize, temperature):
    r = np.random.default_rng(2)
    x, tokens, t = 2 * r.normal(size=9), [3, 8, 3, -1, 0, 11], r.normal(size=6) - 2
    _, dx, _, _, _ = D.distill(x, tokens, t, temperature, normalize)
    for i in range(9):
        e = np.zeros(9)
        e[i] = 1e-6
        diff = (D.distill(x + e, tokens, t, temperature, normalize)[0] - D.distill(x - e, tokens, t, temperature, normalize)[0]) / 2e-6
        assert diff == pytest.approx(dx[i], abs=1e-8, rel=1e-6)


def test_distillation_by_hand():
    # a teacher that agrees with the student over all tokens: no loss, no gradient
    x = np.array([0.3, -1.0, 2.0])
    loss, dx, _, _, _ = D.distill(x, [0, 1, 2], x, 1.7, True)
    assert loss == pytest.approx(0.0, abs=1e-15) and np.allclose(dx, 0.0)
    # one token: cross entropy
    loss, dx, lse, _, _ = D.distill(x, [2], [5.0], 1.0, True)
    assert loss == pytest.approx(lse - 2.0) and np.allclose(dx, np.exp(x - lse) - [0, 0, 1])
    assert D.distill(x, [-1, 3], [1.0, 1.0], 1.0, True)[0] == 0.0
