"""Attention of a chunk of new tokens over a paged cache against the FP64 definition.

Tolerances.  A score is an FP32 sum of `dim` products: off by at most (dim + 8) 2^-23 scale sum |q||k| (the factor two above
2^-24: the accumulators of the tensor cores truncate), which with 2^-20 for the exponential is the relative error of a
weight; a weight may be rounded to the 16-bit type before it meets a value.  So |err(out)| <= u |out| + sum_j p_j |v_j|
(2 (u + e) ) with u the half-unit of the type, e the error of a weight; the factor two covers numerator and sum.  Running
sums over n keys in tiles add at most 2^-20 of the same magnitude.  err(lse) <= e + 2^-22 |lse|."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

from test_gpu_norm_rope import make_cache

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
UNIT = {t: torch.finfo(t).eps / 2 for t in (F16, BF16)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def fill(rng, k, v, kv, table, page, scale=1.0):
    """Random keys and values where a sequence has them; NaN everywhere else."""
    k.fill_(float("nan"))
    v.fill_(float("nan"))
    for b, n in enumerate(kv):
        for j0 in range(0, n, page):
            m = min(page, n - j0)
            for c in (k, v):
                x = torch.from_numpy(scale * rng.standard_normal((m,) + tuple(c.shape[2:])).astype(np.float32))
                c[int(table[b, j0 // page]), :m] = x.to(c.dtype).cuda()


def check(seqs, hq, hk, dim, page, dtype, causal=True, window=-1, order="thd", scale=None, gain=1.0, q_pad=0, hint=None, seed=0):
    rng = np.random.default_rng(seed + dim + 7 * page)
    k, v, cu, kv, table = make_cache(rng, seqs, hk, dim, page, dtype, order)
    fill(rng, k, v, kv, table, page)
    n = int(cu[-1])
    q = torch.from_numpy(gain * rng.standard_normal((n, hq * dim + q_pad)).astype(np.float32)).to(dtype).cuda()
    q = q[:, :hq * dim].unflatten(1, (hq, dim))
    out = torch.full((n, hq, dim), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((n, hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mq, mk = hint or (max(a for a, _ in seqs), max(b for _, b in seqs))
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    ws = A.attention_workspace()
    cache = A.PagedCache(k, v)
    A.paged_attention(cache, q, out, *dev, ws, mq, mk, scale=scale, causal=causal, window=window, lse=lse, status=status)
    first = (out.clone(), lse.clone())
    A.paged_attention(cache, q, out, *dev, ws, mq, mk, scale=scale, causal=causal, window=window, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert torch.equal(first[0], out) and torch.equal(first[1], lse)          # the same bits again
    s = scale or dim ** -0.5
    want, want_lse, mag, smag = O.paged_attention(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(),
                                                  cu, kv, table, s, causal, window)
    u = UNIT[dtype]
    e = (dim + 8) * 2.0 ** -23 * smag + 2.0 ** -20
    tol = u * np.abs(want) + mag * (2 * (u + e[..., None]) + 2.0 ** -20) + 2.0 ** -24
    got = out.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), bad.shape, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])
    got = lse.double().cpu().numpy()
    none = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got), none)
    w = want_lse[~none]
    assert np.all(np.abs(got[~none] - w) <= e[~none] + 2.0 ** -22 * np.abs(w)), np.abs(got[~none] - w).max()


CASES = {
    "one_key": dict(seqs=[(1, 1)], hq=4, hk=1, dim=128, page=16, dtype=BF16),
    "step": dict(seqs=[(1, 37)], hq=8, hk=2, dim=128, page=16, dtype=F16),
    "step_long": dict(seqs=[(1, 5003)], hq=4, hk=1, dim=128, page=16, dtype=BF16),
    "steps_uneven": dict(seqs=[(1, 1), (1, 300), (1, 127), (1, 128), (1, 129), (1, 2000), (1, 16)], hq=8, hk=2, dim=128, page=16, dtype=BF16),
    "drafts": dict(seqs=[(4, 1000), (3, 260), (4, 4)], hq=16, hk=2, dim=128, page=64, dtype=BF16),
    "lengths_of_zero": dict(seqs=[(0, 0), (0, 40), (2, 50), (0, 0), (1, 1), (0, 7)], hq=4, hk=2, dim=64, page=8, dtype=F16),
    "more_new_than_keys": dict(seqs=[(5, 3), (4, 0), (2, 90)], hq=4, hk=2, dim=64, page=16, dtype=BF16),
    "prompt": dict(seqs=[(150, 150)], hq=2, hk=2, dim=128, page=16, dtype=BF16),
    "prompt_wide_tiles": dict(seqs=[(300, 700)], hq=4, hk=1, dim=128, page=32, dtype=BF16),
    "chunks": dict(seqs=[(70, 400), (1, 200), (0, 3), (33, 33), (129, 600)], hq=4, hk=4, dim=128, page=16, dtype=F16),
    "chunks_d64": dict(seqs=[(70, 400), (200, 333)], hq=6, hk=2, dim=64, page=24, dtype=F16),
    "seven_heads_to_one": dict(seqs=[(40, 300), (3, 90)], hq=14, hk=2, dim=64, page=16, dtype=BF16),
    "dim_96": dict(seqs=[(20, 150), (1, 70)], hq=4, hk=2, dim=96, page=16, dtype=BF16),
    "dim_80": dict(seqs=[(130, 260)], hq=4, hk=4, dim=80, page=128, dtype=F16),
    "dim_32": dict(seqs=[(9, 140)], hq=4, hk=4, dim=32, page=16, dtype=F16),
    "dim_40": dict(seqs=[(9, 140), (1, 300)], hq=2, hk=1, dim=40, page=16, dtype=BF16),
    "dim_256": dict(seqs=[(5, 90), (1, 300)], hq=2, hk=1, dim=256, page=16, dtype=BF16),
    "all_keys": dict(seqs=[(20, 150), (1, 70), (3, 2)], hq=4, hk=2, dim=128, page=16, dtype=BF16, causal=False),
    "window": dict(seqs=[(150, 400), (1, 900), (4, 130)], hq=4, hk=2, dim=128, page=16, dtype=BF16, window=100),
    "window_zero": dict(seqs=[(50, 200), (1, 300)], hq=4, hk=2, dim=64, page=16, dtype=F16, window=0),
    "window_all_keys": dict(seqs=[(50, 200)], hq=4, hk=2, dim=64, page=16, dtype=F16, window=20, causal=False),
    "page_of_300": dict(seqs=[(20, 700), (1, 301)], hq=4, hk=2, dim=128, page=304, dtype=BF16),
    "page_of_5": dict(seqs=[(20, 70), (1, 31)], hq=4, hk=2, dim=128, page=5, dtype=BF16),
    "page_of_1": dict(seqs=[(3, 33)], hq=2, hk=1, dim=64, page=1, dtype=BF16),
    "rows_steps": dict(seqs=[(1, 300), (1, 1), (1, 1000), (3, 129), (0, 12)], hq=8, hk=2, dim=128, page=5, dtype=BF16),
    "rows_prompt": dict(seqs=[(300, 700), (70, 400)], hq=4, hk=2, dim=128, page=20, dtype=F16),
    "rows_prompt_long": dict(seqs=[(130, 3000), (1, 2500)], hq=4, hk=2, dim=128, page=100, dtype=BF16),
    "rows_dim_96": dict(seqs=[(130, 260), (1, 70)], hq=4, hk=2, dim=96, page=12, dtype=BF16),
    "rows_dim_64": dict(seqs=[(20, 600), (16, 40)], hq=8, hk=2, dim=64, page=3, dtype=F16),
    "rows_dim_40": dict(seqs=[(90, 140), (1, 300)], hq=2, hk=1, dim=40, page=1, dtype=BF16),
    "rows_window": dict(seqs=[(150, 400), (1, 900), (4, 130)], hq=4, hk=2, dim=128, page=12, dtype=BF16, window=100, order="htd"),
    "heads_outer": dict(seqs=[(20, 170), (1, 310)], hq=4, hk=2, dim=128, page=16, dtype=BF16, order="htd"),
    "odd_query_stride": dict(seqs=[(5, 90)], hq=3, hk=3, dim=64, page=16, dtype=BF16, q_pad=3),
    "padded_query_rows": dict(seqs=[(5, 90), (140, 141)], hq=3, hk=3, dim=64, page=16, dtype=BF16, q_pad=64),
    "sharp": dict(seqs=[(60, 500), (1, 900)], hq=4, hk=2, dim=128, page=16, dtype=F16, gain=12.0),
    "sharp_bf16": dict(seqs=[(60, 500), (1, 900)], hq=4, hk=2, dim=128, page=16, dtype=BF16, gain=40.0),
    "flat": dict(seqs=[(60, 500), (1, 900)], hq=4, hk=2, dim=128, page=16, dtype=F16, gain=0.01),
    "own_scale": dict(seqs=[(10, 100)], hq=4, hk=2, dim=128, page=16, dtype=BF16, scale=0.3),
    "short_hints": dict(seqs=[(200, 500), (1, 300)], hq=4, hk=2, dim=128, page=16, dtype=BF16, hint=(1, 1)),
    "long_hints": dict(seqs=[(1, 500), (1, 300)], hq=4, hk=2, dim=128, page=16, dtype=BF16, hint=(4096, 100000)),
    "one_head_many_rows": dict(seqs=[(3, 1500)], hq=100, hk=1, dim=128, page=16, dtype=BF16),
    "group_over_a_tile": dict(seqs=[(2, 150)], hq=160, hk=1, dim=64, page=16, dtype=BF16),
    "many_sequences": dict(seqs=[(i % 3, 1 + (37 * i) % 200) for i in range(333)], hq=2, hk=1, dim=64, page=16, dtype=BF16),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    check(**CASES[name])


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 513])
def test_every_length_around_a_tile(n):
    check([(1, n), (min(n, 3), n), (n, n)], 2, 1, 64, 16, BF16, seed=n)


def test_no_new_tokens():
    k = torch.zeros(2, 16, 1, 64, dtype=BF16, device="cuda")
    q = torch.zeros(0, 2, 64, dtype=BF16, device="cuda")
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    A.paged_attention(A.PagedCache(k, k.clone()), q, q.clone(), z, z[:1], z[:1, None], A.attention_workspace(), 0, 0)
    torch.cuda.synchronize()


def test_infinite_scores_and_nan_keys_stay_in_their_sequence():
    """A NaN among a sequence's visible keys makes its rows NaN; the other sequences do not see it."""
    rng = np.random.default_rng(2)
    k, v, cu, kv, table = make_cache(rng, [(1, 200), (1, 300), (1, 100)], 1, 128, 16, BF16, "thd")
    fill(rng, k, v, kv, table, 16)
    k[int(table[1, 3]), 5] = float("nan")
    q = torch.randn(3, 2, 128, device="cuda").to(BF16)
    out = torch.zeros_like(q)
    A.paged_attention(A.PagedCache(k, v), q, out, *(torch.from_numpy(x).cuda() for x in (cu, kv, table)), A.attention_workspace(), 1, 300)
    assert out.isnan().any(-1).any(-1).tolist() == [False, True, False]


@pytest.mark.parametrize("what", ["query heads", "tokens"])
def test_expanded_dimensions(what):
    """An expanded dimension (stride 0) of the queries gives what its copies give; a cache, which is written to, has none."""
    rng = np.random.default_rng(3)
    seqs, hq, hk, dim, page = [(40, 300), (1, 70)], 4, 2, 64, 16
    k, v, cu, kv, table = make_cache(rng, seqs, hk, dim, page, BF16, "thd")
    fill(rng, k, v, kv, table, page)
    n = int(cu[-1])
    q = torch.from_numpy(rng.standard_normal((n, hq, dim)).astype(np.float32)).to(BF16).cuda()
    if what == "query heads": q = q[:, :1].expand(n, hq, dim)
    if what == "tokens": q = q[:1].expand(n, hq, dim)
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    ws = A.attention_workspace()
    out = torch.full((n, hq, dim), 7.0, dtype=BF16, device="cuda")
    A.paged_attention(A.PagedCache(k, v), q, out, *dev, ws, 40, 300)
    torch.cuda.synchronize()
    s = dim ** -0.5
    want, _, mag, smag = O.paged_attention(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(),
                                           cu, kv, table, s, True, -1)
    u, e = UNIT[BF16], (dim + 8) * 2.0 ** -23 * smag + 2.0 ** -20
    tol = u * np.abs(want) + mag * (2 * (u + e[..., None]) + 2.0 ** -20) + 2.0 ** -24
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    for pair in ((k[:, :, :1].expand(k.shape), v), (k, v[:, :, :1].expand(v.shape))):
        with pytest.raises(fpsk.FpskError):
            A.paged_attention(A.PagedCache(*pair), q, out, *dev, ws, 40, 300)


@pytest.mark.parametrize("page", [16, 12])
def test_pages_outside_the_cache_are_reported(page):
    rng = np.random.default_rng(2)
    k, v, cu, kv, table = make_cache(rng, [(1, 200), (1, 100)], 1, 128, page, BF16, "thd")
    fill(rng, k, v, kv, table, page)
    table[0, 4] = 12345
    q = torch.randn(2, 2, 128, device="cuda").to(BF16)
    out = torch.zeros_like(q)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_attention(A.PagedCache(k, v), q, out, *(torch.from_numpy(x).cuda() for x in (cu, kv, table)), A.attention_workspace(), 1, 200, status=status)
    assert int(status) == fpsk.ERR_PARAM
    assert not out[1].isnan().any()


def test_other_stream_and_graph_replay():
    rng = np.random.default_rng(9)
    k, v, cu, kv, table = make_cache(rng, [(1, 700), (1, 90)], 2, 128, 16, BF16, "thd")
    fill(rng, k, v, kv, table, 16)
    q = torch.randn(2, 8, 128, device="cuda").to(BF16)
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    ws, cache = A.attention_workspace(), A.PagedCache(k, v)
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    A.paged_attention(cache, q, out, *dev, ws, 1, 700)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    A.paged_attention(cache, q, again, *dev, ws, 1, 700, stream=st)
    st.synchronize()
    assert torch.equal(out, again)
    again.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.paged_attention(cache, q, again, *dev, ws, 1, 700)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, again)


def test_refusals():
    k = torch.zeros(2, 16, 2, 64, dtype=BF16, device="cuda")
    cache = A.PagedCache(k, k.clone())
    q = torch.zeros(1, 4, 64, dtype=BF16, device="cuda")
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = A.attention_workspace()
    dev = (z, z[:1], z[:1, None])
    with pytest.raises(ValueError):
        A.paged_attention(cache, q.half(), q.clone(), *dev, ws, 1, 1)
    with pytest.raises(ValueError):
        A.paged_attention(cache, q, q[:, :2].clone(), *dev, ws, 1, 1)
    with pytest.raises(ValueError):
        A.paged_attention(cache, q, q.clone(), *dev, ws, 1, 1, scale=float("nan"))
    for heads in (3, 5):
        x = torch.zeros(1, heads, 64, dtype=BF16, device="cuda")
        with pytest.raises(fpsk.FpskError) as e:
            A.paged_attention(cache, x, x.clone(), *dev, ws, 1, 1)
        assert e.value.status == fpsk.ERR_SHAPE
    with pytest.raises(fpsk.FpskError) as e:
        A.paged_attention(cache, q, q.clone(), *dev, ws, 1, 1, window=-2)
    assert e.value.status == fpsk.ERR_PARAM
    with pytest.raises(fpsk.FpskError) as e:
        A.paged_attention(cache, q, q.clone(), *dev, ws[:128], 1, 1)
    assert e.value.status == fpsk.ERR_WORKSPACE
    with pytest.raises(fpsk.FpskError) as e:
        A.paged_attention(cache, q, q.clone(), *dev, ws[1:], 1, 1)
    assert e.value.status == fpsk.ERR_ALIGN
