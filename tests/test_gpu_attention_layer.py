"""The verified attention layer end to end: prompts and decoding steps over the paged cache give what a plain layer in 64 bits gives
for the whole sequences, clean products stay clean, a corrupted accumulator entry is reported."""
import pytest
import torch

from paper_2609_19758_b200 import attention_layer as L
from paper_2609_19758_b200 import build as B

pytestmark = pytest.mark.gpu


def _plain_layer(layer, x):
    """Outputs of one sequence in 64 bits from its inputs (tokens, hidden)."""
    hq, hk, dim = layer.hq, layer.hk, layer.dim
    n = x.shape[0]
    c = x.double() @ layer.qkv_weight.double()
    q, k, v = (t.unflatten(1, (-1, dim)) for t in c.split((hq * dim, hk * dim, hk * dim), dim=1))
    cos, sin = layer.cos[:n].double()[:, None], layer.sin[:n].double()[:, None]

    def head(t, w):
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + layer.eps) * w.double()
        a, b = t[..., :dim // 2], t[..., dim // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    q, k = head(q, layer.q_weight), head(k, layer.k_weight)
    k, v = (t.repeat_interleave(hq // hk, 1) for t in (k, v))
    s = torch.einsum("ihd,jhd->hij", q, k) * dim ** -0.5
    s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=x.device).triu(1), float("-inf"))
    out = torch.einsum("hij,jhd->ihd", s.softmax(-1), v)
    return out.flatten(1) @ layer.out_weight.double()


@pytest.mark.parametrize("hidden,hq,hk,dim,prompts,dtype", [(512, 8, 2, 64, (70, 1, 33), torch.float16), (1024, 8, 8, 128, (200, 5), torch.bfloat16)])
def test_layer_equals_the_plain_layer(hidden, hq, hk, dim, prompts, dtype):
    B.build()
    r = L.demo(hidden, hq, hk, dim, prompts, steps=3, dtype=dtype, seed=1)
    assert not any(r["fired"])
    assert r["fired_on_fault"]
    # Roundings to 16 bits (unit u) on the way: q and k move a score by about u sqrt(2) |q||k| / sqrt(dim) (|q| = |k| = sqrt(dim), so
    # u sqrt(2 dim) at most), v, the weights and the layer's middle by u each; the output is a sum of hq dim such terms of unit size.
    u = torch.finfo(dtype).eps / 2
    for x, y in zip(r["inputs"], r["outputs"]):
        want = _plain_layer(r["layer"], x)[:-1]                        # (the last token's accumulator was corrupted)
        err = float((y[:-1].double() - want).norm() / want.norm())
        assert err <= u * (2 * dim) ** 0.5 + 4 * u, err
