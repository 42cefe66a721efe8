"""FP64 definitions of the operators on a decoder's output projection and head, in plain numpy, one row at a time.

Shares no code with the GPU path.  Next to the values stand the sums of magnitudes that their rounding errors scale with, so that
a test can derive its tolerance from the inputs.
"""
from __future__ import annotations

import numpy as np

E4M3_TOP = 448.0


def add_norm(x, residual, w, eps):
    """Rows of h = x + residual and of y = h / sqrt(mean(h^2) + eps) w."""
    h = np.asarray(x, dtype=np.float64) + (0.0 if residual is None else np.asarray(residual, dtype=np.float64))
    y = np.empty_like(h)
    for t in range(h.shape[0]):
        y[t] = h[t] / np.sqrt(np.mean(h[t] ** 2) + eps) * (1.0 if w is None else w)
    return h, y


def e4m3_scales(y, group):
    """max |y| / 448 of every group of a row; 1 for zeros."""
    dim = y.shape[1]
    width = group or dim
    starts = range(0, dim, width)
    s = np.empty((y.shape[0], len(starts)))
    for t in range(y.shape[0]):
        for i, c in enumerate(starts):
            top = np.abs(y[t, c:c + width]).max()
            s[t, i] = max(top / E4M3_TOP, 2.0 ** -126) if top > 0 else 1.0
    return s


def add_norm_grad(h, w, dy, dh, eps):
    """Gradients of sum(dy * y) + sum(dh * h) with respect to h and w, and the magnitudes of their terms."""
    h, dy = np.asarray(h, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dim = h.shape[1]
    w = np.ones(dim) if w is None else w
    dx, mag = np.empty_like(h), np.empty_like(h)
    dw, dw_mag = np.zeros(dim), np.zeros(dim)
    for t in range(h.shape[0]):
        r = 1.0 / np.sqrt(np.mean(h[t] ** 2) + eps)
        # y_i = h_i r w_i, dr/dh_j = - r^3 h_j / dim
        g = dy[t] * w
        dx[t] = g * r - (g @ h[t]) * r ** 3 * h[t] / dim
        mag[t] = np.abs(g) * r + (np.abs(g) @ np.abs(h[t])) * r ** 3 * np.abs(h[t]) / dim
        if dh is not None:
            dx[t] += dh[t]
            mag[t] += np.abs(dh[t])
        dw += dy[t] * h[t] * r
        dw_mag += np.abs(dy[t] * h[t] * r)
    return dx, mag, dw, dw_mag


def adjust_logits(row, history=(), n_prompt=0, repetition=1.0, frequency=0.0, presence=0.0, biases=(), allowed=None):
    """One row of logits: z, and the magnitude that its rounding errors scale with.  biases: (token, value) pairs; allowed: booleans."""
    z = np.array(row, dtype=np.float64)
    mag = np.abs(z)
    seen, made = {}, {}
    for i, v in enumerate(history):
        if 0 <= v < len(z):
            seen[v] = True
            if i >= n_prompt:
                made[v] = made.get(v, 0) + 1
    for v in seen:
        z[v] = z[v] / repetition if z[v] > 0 else z[v] * repetition
        mag[v] = max(mag[v], abs(z[v]))
    for v, c in made.items():
        z[v] -= frequency * c + presence
        mag[v] += 2 * (abs(frequency) * c + abs(presence))
    for v, value in biases:
        if 0 <= v < len(z):
            z[v] += value
            mag[v] += 2 * abs(value)
    if allowed is not None:
        z[~np.asarray(allowed)] = -np.inf
    return z, mag


def log_sum_exp(z):
    top = z.max()
    return top if np.isinf(top) else top + np.log(np.exp(z - top).sum())


def distill(row, tokens, teacher, temperature, normalize):
    """One row: loss, gradient with respect to the logits, lse of logits / temperature, and the magnitudes (of the loss's terms; m q and p
    of the gradient)."""
    x = np.asarray(row, dtype=np.float64) / temperature
    lse = log_sum_exp(x)
    q = np.exp(x - lse)
    entries = [(int(v), float(t)) for v, t in zip(tokens, teacher) if 0 <= v < len(x) and t != -np.inf]
    if not entries:
        return 0.0, np.zeros(len(x)), lse, 0.0, np.zeros(len(x))
    t = np.array([e[1] for e in entries])
    logp = t / temperature - log_sum_exp(t / temperature) if normalize else t
    p = np.zeros(len(x))
    loss, mag = 0.0, 0.0
    for (v, tv), lp in zip(entries, logp):
        loss += np.exp(lp) * (lp - (x[v] - lse))
        mag += np.exp(lp) * (abs(lp) + abs(tv) + abs(x[v]) + abs(lse) + 1.0)
        p[v] += np.exp(lp)
    m = p.sum()
    return loss, (m * q - p) / temperature, lse, mag, (m * q + p) / temperature
