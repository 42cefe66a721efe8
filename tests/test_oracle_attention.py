"""The FP64 definitions of the attention operators against differences and against closed forms (CPU)."""
import numpy as np
import pytest

from oracle import attention_oracle as A


def _tables(rng, tokens, rot):
    a = rng.uniform(0, 6, (tokens, rot // 2))
    return np.cos(a), np.sin(a)


@pytest.mark.parametrize("dim,rot,interleaved,normed", [(16, 16, False, True), (24, 8, False, True), (16, 16, True, True),
                                                         (24, 16, True, False), (8, 0, False, True)])
def test_gradient_equals_differences(dim, rot, interleaved, normed):
    rng = np.random.default_rng(dim + rot)
    x, dy = rng.standard_normal((3, 2, dim)), rng.standard_normal((3, 2, dim))
    w = 1 + 0.3 * rng.standard_normal(dim) if normed else None
    c, s = _tables(rng, 3, rot)
    eps = 1e-3

    def f(x_, w_):
        return float(np.sum(dy * A.norm_rope(x_, w_, c, s, rot, eps, interleaved)[0]))

    dx, _, dw, _ = A.norm_rope_grad(x, w, dy, c, s, rot, eps, interleaved)
    h = 1e-5                                     # central differences: truncation O(h^2), cancellation 1e-16 / h
    for idx in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[idx] = h
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * h) - dx[idx]) < 1e-7
    if normed:
        for i in range(dim):
            d = np.zeros(dim)
            d[i] = h
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * h) - dw[i]) < 1e-7


def test_rotation_is_orthogonal_and_depends_on_the_distance_alone():
    rng = np.random.default_rng(1)
    for inter in (False, True):
        q, k = rng.standard_normal(32), rng.standard_normal(32)
        inv = 10000.0 ** (-np.arange(12) / 12)
        dots = []
        for p in (0, 5, 900):
            rq = A.rotate(q, np.cos((p + 7) * inv), np.sin((p + 7) * inv), 24, inter)
            rk = A.rotate(k, np.cos(p * inv), np.sin(p * inv), 24, inter)
            back = A.rotate(rq, np.cos((p + 7) * inv), np.sin((p + 7) * inv), 24, inter, inverse=True)
            assert np.allclose(back, q, atol=1e-12)
            dots.append(rq @ rk)
        assert np.allclose(dots, dots[0], atol=1e-10)


def test_attention_closed_forms():
    # equal scores: the mean of the visible values; one key: that value; none: zero and -inf
    page, dim = 4, 8
    k = np.zeros((4, page, 1, dim))
    v = np.arange(4 * page * dim, dtype=np.float64).reshape(4, page, 1, dim)
    table = np.array([[2, 0, -1], [1, -1, -1], [3, -1, -1]])
    q = np.ones((6, 2, dim))
    cu, kv = [0, 2, 3, 6], [7, 1, 2]             # the third sequence has three new tokens and two keys
    out, lse, _, _ = A.paged_attention(q, k, v, cu, kv, table, 0.5)
    flat = np.concatenate([v[2, :, 0], v[0, :, 0]])
    assert np.allclose(out[0, 0], flat[:6].mean(0)) and np.allclose(out[1, 1], flat[:7].mean(0))
    assert np.allclose(lse[1], np.log(7)) and np.allclose(out[2, 0], v[1, 0, 0])
    assert np.all(out[3] == 0) and np.all(np.isneginf(lse[3])) and np.allclose(out[4, 0], v[3, 0, 0])
    win, _, _, _ = A.paged_attention(q, k, v, cu, kv, table, 0.5, window=2)
    assert np.allclose(win[1, 0], flat[4:7].mean(0))
    full, _, _, _ = A.paged_attention(q, k, v, cu, kv, table, 0.5, causal=False)
    assert np.allclose(full[0, 0], flat[:7].mean(0))
