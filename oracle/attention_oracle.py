"""FP64 definitions of the attention operators beside a verified projection, in plain numpy, one head vector at a time.

Shares no code with the GPU path.  Next to every value stands the sum of magnitudes that its rounding errors scale
with, so that a test can derive its tolerance from the inputs.
"""
from __future__ import annotations

import numpy as np


def pair_channels(dim: int, rot: int, interleaved: bool):
    """Channel pairs (first, second) of the rotation."""
    if interleaved:
        return [(2 * i, 2 * i + 1) for i in range(rot // 2)]
    return [(i, i + rot // 2) for i in range(rot // 2)]


def rotate(z, c, s, rot, interleaved, inverse=False):
    """Rotation of one head vector; c, s: rot / 2 factors."""
    y = np.array(z, dtype=np.float64)
    for i, (a, b) in enumerate(pair_channels(len(z), rot, interleaved)):
        si = -s[i] if inverse else s[i]
        y[a] = z[a] * c[i] - z[b] * si
        y[b] = z[b] * c[i] + z[a] * si
    return y


def pair_magnitude(z, rot, interleaved):
    """|z_a| + |z_b| for the channels of a pair, |z| for the others."""
    y = np.abs(z)
    for a, b in pair_channels(len(z), rot, interleaved):
        y[a] = y[b] = abs(z[a]) + abs(z[b])
    return y


def norm_rope(x, w, c, s, rot, eps, interleaved=False):
    """x (tokens, heads, dim); w (dim,) or None; c, s (tokens, rot / 2) of the tokens' positions.  Returns y and its
    magnitudes."""
    x = np.asarray(x, dtype=np.float64)
    y, mag = np.empty_like(x), np.empty_like(x)
    for t in range(x.shape[0]):
        for h in range(x.shape[1]):
            z = x[t, h]
            if w is not None:
                z = z / np.sqrt(np.mean(z * z) + eps) * w
            y[t, h] = rotate(z, c[t], s[t], rot, interleaved)
            mag[t, h] = pair_magnitude(z, rot, interleaved)
    return y, mag


def norm_rope_grad(x, w, dy, c, s, rot, eps, interleaved=False):
    """Gradients of sum(dy * norm_rope(x)) with respect to x and w, and the magnitudes of their terms."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    dx, mag = np.empty_like(x), np.empty_like(x)
    dw, dw_mag = np.zeros(x.shape[2]), np.zeros(x.shape[2])
    for t in range(x.shape[0]):
        for h in range(x.shape[1]):
            u = rotate(dy[t, h], c[t], s[t], rot, interleaved, inverse=True)
            um = pair_magnitude(dy[t, h], rot, interleaved)
            if w is None:
                dx[t, h], mag[t, h] = u, um
                continue
            r = 1.0 / np.sqrt(np.mean(x[t, h] ** 2) + eps)
            n = x[t, h] * r
            g = u * w
            dx[t, h] = r * (g - n * np.mean(g * n))
            mag[t, h] = r * (um * np.abs(w) + np.abs(n) * np.mean(um * np.abs(w) * np.abs(n)))
            dw += u * n
            dw_mag += um * np.abs(n)
    return dx, mag, dw, dw_mag


def places(cu_q, kv_len, page_size, block_table):
    """(sequence, position, page, row) of every new token; position < 0: no place (page -1)."""
    out = []
    for b in range(len(kv_len)):
        for t in range(cu_q[b], cu_q[b + 1]):
            p = kv_len[b] - (cu_q[b + 1] - t)
            out.append((b, p, int(block_table[b][p // page_size]) if p >= 0 else -1, p % page_size))
    return out


def visible(p, kv_len, causal, window):
    """The keys [lo, hi) that the token at position p sees."""
    if p < 0:
        return 0, 0
    hi = min(p + 1, kv_len) if causal else kv_len
    lo = max(0, p - window) if window >= 0 else 0
    return lo, max(lo, hi)


def paged_attention(q, k_cache, v_cache, cu_q, kv_len, block_table, scale, causal=True, window=-1):
    """q (tokens, query heads, dim); caches (pages, page size, key heads, dim).  Returns out, lse, sum_j p_j |v_j|, and
    the largest scale sum |q| |k| of each row."""
    n, hq, dim = q.shape
    page, hk = k_cache.shape[1], k_cache.shape[2]
    out, mag = np.zeros((n, hq, dim)), np.zeros((n, hq, dim))
    lse, smag = np.full((n, hq), -np.inf), np.zeros((n, hq))
    for t, (b, p, _, _) in enumerate(places(cu_q, kv_len, page, np.maximum(block_table, 0))):
        lo, hi = visible(p, kv_len[b], causal, window)
        if hi <= lo:
            continue
        j = np.arange(lo, hi)
        pg, row = np.asarray(block_table[b])[j // page], j % page
        for h in range(hq):
            k = k_cache[pg, row, h // (hq // hk)].astype(np.float64)
            v = v_cache[pg, row, h // (hq // hk)].astype(np.float64)
            s = scale * (k @ q[t, h].astype(np.float64))
            top = s.max()
            e = np.exp(s - top)
            out[t, h] = (e @ v) / e.sum()
            mag[t, h] = (e @ np.abs(v)) / e.sum()
            lse[t, h] = top + np.log(e.sum())
            smag[t, h] = scale * (np.abs(k) @ np.abs(q[t, h].astype(np.float64))).max()
    return out, lse, mag, smag
