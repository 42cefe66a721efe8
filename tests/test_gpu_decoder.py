"""The decoder's operators together: layers joined by the residual norm, greedy tokens under penalties and masks, a dirty step repeated,
and a training step of the head, against plain computations in 64 bits."""
import pytest
import torch

from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import decoder as M

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def plain_states(d, tokens):
    """The last states of one sequence in 64 bits."""
    n = len(tokens)
    h = d.embedding[torch.tensor(tokens, device="cuda")].double()

    def normed(h, w):
        return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + d.eps) * w.double()

    x = normed(h, d.norm_weights[0])
    for layer, weight in zip(d.layers, d.norm_weights[1:]):
        hq, hk, dim = layer.hq, layer.hk, layer.dim
        q, k, v = (t.unflatten(1, (-1, dim)) for t in (x @ layer.qkv_weight.double()).split((hq * dim, hk * dim, hk * dim), dim=1))
        cos, sin = layer.cos[:n].double()[:, None], layer.sin[:n].double()[:, None]

        def head(t, w):
            t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + layer.eps) * w.double()
            a, b = t[..., :dim // 2], t[..., dim // 2:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        q, k = head(q, layer.q_weight), head(k, layer.k_weight)
        k, v = (t.repeat_interleave(hq // hk, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) * dim ** -0.5
        s.masked_fill_(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
        h = h + torch.einsum("hij,jhd->ihd", s.softmax(-1), v).flatten(1) @ layer.out_weight.double()
        x = normed(h, weight)
    return x


@pytest.mark.parametrize("dtype,layers", [(torch.float16, 1), (torch.bfloat16, 3)])
def test_states_equal_the_plain_decoder(dtype, layers):
    d = M.demo_decoder(vocab=600, hidden=512, layers=layers, hq=4, hk=2, dim=64, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(0)
    prompts = [torch.randint(0, 600, (n,), generator=g).tolist() for n in (37, 1, 150)]
    seqs = [d.open() for _ in prompts]
    x = d.step(torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda"), seqs, [len(p) for p in prompts])
    more = [[5], [7], [9]]
    y = d.step(torch.tensor([5, 7, 9], dtype=torch.int32, device="cuda"), seqs, [1, 1, 1])
    assert not d.fired()
    # Roundings to 16 bits (u) on the way of a layer: its input, q and k (which move a score by u sqrt(2 dim) at most, see the layer's own
    # test), v, the weights, the middle: u (4 + sqrt(2 dim)) of the layer's unit output, added to a stream of size 1 and more that is rounded
    # once (u); the layers' errors add up, and pass through the layers behind with a factor that the unit weights keep near 1: 2 covers it.
    u = torch.finfo(dtype).eps / 2
    bound = 2 * layers * u * (6 + (2 * 64) ** 0.5) + u
    for p, m, xs, ys in zip(prompts, more, x.split([len(p) for p in prompts]), y.split(1)):
        want = plain_states(d, p + m)
        err = float((torch.cat([xs, ys]).double() - want).norm() / want.norm())
        assert err <= bound, (err, bound)


def test_greedy_tokens_follow_the_penalties_and_masks():
    d = M.demo_decoder(vocab=1000, hidden=512, layers=2, hq=4, hk=2, dim=64, seed=4)
    prompts = [[1, 2, 3, 1, 1], [999]]
    free = d.generate(prompts, 6)
    assert all(len(t) == 6 and all(0 <= v < 1000 for v in t) for t in free)
    # a frequency that nothing outweighs: no token comes twice
    once = d.generate(prompts, 6, frequency=1e4)
    assert all(len(set(t)) == 6 for t in once) and [t[0] for t in once] == [t[0] for t in free]
    # only these
    mask = torch.zeros(32, dtype=torch.int32, device="cuda")
    mask[3], mask[10] = 1 << 4, 1 << 30
    held = d.generate(prompts, 3, presence=1e4, mask=mask)
    assert all(t[0] in (100, 350) and t[1] in (100, 350) and t[0] != t[1] for t in held)


def test_a_dirty_step_is_repeated():
    d = M.demo_decoder(vocab=1000, hidden=512, layers=2, hq=4, hk=2, dim=64, seed=5)
    prompts = [list(range(20)), [3, 4]]
    plain = d.generate(prompts, 4, repetition=1.3)
    free = [list(layer.pages.free) for layer in d.layers]
    assert d.generate(prompts, 4, repetition=1.3, fault_at=0) == plain
    assert d.generate(prompts, 4, repetition=1.3, fault_at=2) == plain
    # every page is back
    assert [sorted(f) for f in free] == [sorted(layer.pages.free) for layer in d.layers] and all(len(f) == 256 for f in free)


def test_a_refused_step_changes_nothing():
    d = M.demo_decoder(vocab=100, hidden=256, layers=2, hq=2, hk=2, dim=64, seed=6)
    seq = d.open()
    d.step(torch.arange(5, dtype=torch.int32, device="cuda"), [seq], [5])
    with pytest.raises(ValueError):
        d.step(torch.arange(5, dtype=torch.int32, device="cuda"), [seq], [6])
    d.layers[1].pages.free, kept = [], d.layers[1].pages.free          # the second layer's cache is full: the first takes its step back
    with pytest.raises(RuntimeError):
        d.step(torch.arange(20, dtype=torch.int32, device="cuda"), [seq], [20])
    d.layers[1].pages.free = kept
    assert [layer.pages.length for layer in d.layers] == [[5], [5]]
    for bad in ([], [[]], [[100]], [[-1]]):
        with pytest.raises(ValueError):
            d.generate(bad, 1)
    with pytest.raises(RuntimeError, match="allows nothing"):
        d.generate([[1]], 2, mask=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert not d.fired()
    d.step(torch.tensor([3, 100], dtype=torch.int32, device="cuda"), [seq], [2])
    with pytest.raises(RuntimeError, match="status 10"):
        d.fired()
    d.retract()
    assert not d.fired() and [layer.pages.length[seq] for layer in d.layers] == [5, 5]
    with pytest.raises(ValueError):
        M.VerifiedDecoder(d.embedding, d.layers, d.norm_weights[:2], d.head)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_distilling_head(dtype):
    """A training step's share of the head against autograd in 64 bits.  The logits' gradient is rounded to 16 bits (u of each entry) and
    the products are FP32: their relative error in norm is at most u, and as much again for sums whose terms cancel is what 2 u allows
    beside the FP32 parts (2^-16 is far above them)."""
    g = torch.Generator(device="cuda").manual_seed(7)
    rows, hidden, vocab, top = 160, 512, 3001 - 1, 24
    head = M.VerifiedHead((torch.randn(hidden, vocab, generator=g, device="cuda") * hidden ** -0.5).to(dtype))
    x = torch.randn(rows, hidden, generator=g, device="cuda").to(dtype)
    token = torch.randint(0, vocab, (rows, top), generator=g, device="cuda", dtype=torch.int32)
    t = 2 * torch.randn(rows, top, generator=g, device="cuda")
    weight = torch.full((rows,), 1.0, device="cuda")
    weight[::7] = 0.0
    loss, dx, dw = head.distill(x, token, t, weight, temperature=1.5)
    assert not head.fired()
    xd, wd = x.double().requires_grad_(), head.weight.double().requires_grad_()
    logq = torch.log_softmax(xd @ wd / 1.5, -1)
    logp = torch.log_softmax(t.double() / 1.5, -1)
    want = (logp.exp() * (logp - logq.gather(1, token.long()))).sum(-1)
    (want * weight.double()).sum().backward()
    u = torch.finfo(dtype).eps / 2
    live = weight != 0
    assert float((loss.double() - want.detach())[live].abs().max()) <= 2.0 ** -16 * float(want.detach().abs().max()) and bool((loss[~live] == 0).all())
    for got, ref in ((dx, xd.grad), (dw, wd.grad)):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2 * u + 2.0 ** -16


def test_command(capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["decoder", "--steps", "3", "--prompts", "4,1"])
    M.main()
    said = capsys.readouterr().out
    assert "the same tokens" in said and said.count("prompt of") == 2
