"""Attention over pages where the scores lie far from zero or far from each other: windows whose keys all score very low (a row
of a tile may see nothing in its item's first steps), and a dominant key above a long tail of small weights.

Tolerances: those of test_gpu_paged_attention.py, whose derivation holds for any scores."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B

from test_gpu_norm_rope import make_cache

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
UNIT = {t: torch.finfo(t).eps / 2 for t in (F16, BF16)}


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def compare(q, k, v, cu, kv, table, mq, mk, causal=True, window=-1):
    n, hq, dim = q.shape
    out = torch.full_like(q, 7.0)
    lse = torch.full((n, hq), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    A.paged_attention(A.PagedCache(k, v), q, out, *dev, A.attention_workspace(), mq, mk, causal=causal, window=window, lse=lse, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    want, want_lse, mag, smag = O.paged_attention(q.double().cpu().numpy(), k.double().cpu().numpy(), v.double().cpu().numpy(),
                                                  cu, kv, table, dim ** -0.5, causal, window)
    u = UNIT[q.dtype]
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


LOW = {  # name: new and present tokens of each sequence, query heads, key heads, dim, page, type, window
    "one_token": dict(seqs=[(1, 900), (1, 131), (1, 70), (1, 260)], hq=4, hk=2, dim=128, page=16, dtype=BF16, window=50),
    "one_token_d64": dict(seqs=[(1, 900), (1, 131), (1, 300)], hq=8, hk=2, dim=64, page=16, dtype=F16, window=37),
    "one_token_long": dict(seqs=[(1, 9000)], hq=8, hk=1, dim=128, page=16, dtype=BF16, window=5003),
    "a_few_tokens": dict(seqs=[(6, 900), (5, 200)], hq=4, hk=1, dim=128, page=16, dtype=BF16, window=100),
    "one_tile_d64": dict(seqs=[(30, 700), (17, 300)], hq=8, hk=2, dim=64, page=16, dtype=BF16, window=75),
    "one_tile_d64_long": dict(seqs=[(30, 4000)], hq=4, hk=1, dim=64, page=16, dtype=F16, window=1000),
    "two_tiles": dict(seqs=[(150, 400), (200, 200), (90, 900)], hq=4, hk=2, dim=128, page=16, dtype=BF16, window=100),
    "two_tiles_f16": dict(seqs=[(150, 400), (131, 900)], hq=2, hk=2, dim=128, page=16, dtype=F16, window=129),
    "two_tiles_d64": dict(seqs=[(200, 333)], hq=6, hk=2, dim=64, page=24, dtype=BF16, window=20),
    "two_tiles_long": dict(seqs=[(140, 6000)], hq=2, hk=1, dim=128, page=16, dtype=BF16, window=3000),
    "all_later_keys": dict(seqs=[(150, 400)], hq=2, hk=1, dim=128, page=16, dtype=BF16, window=65, causal=False),
    "copied_rows": dict(seqs=[(150, 400), (1, 900)], hq=4, hk=2, dim=128, page=12, dtype=BF16, window=100),
    "copied_rows_step": dict(seqs=[(1, 900), (2, 300)], hq=4, hk=2, dim=64, page=5, dtype=F16, window=50),
    # one CTA on all of an item (which a short promise of lengths asks for): a worker, and a quarter of its lanes, has steps before the
    # first that it sees
    "one_token_whole": dict(seqs=[(1, 1400), (1, 1500)], hq=4, hk=1, dim=128, page=16, dtype=BF16, window=777, whole=True),
    "one_token_whole_d64": dict(seqs=[(1, 1400), (3, 1431)], hq=8, hk=1, dim=64, page=16, dtype=F16, window=590, whole=True),
    "one_tile_whole_d64": dict(seqs=[(30, 1700)], hq=4, hk=1, dim=64, page=16, dtype=BF16, window=555, whole=True),
    "one_tile_whole_d64_f16": dict(seqs=[(100, 1700)], hq=1, hk=1, dim=64, page=16, dtype=F16, window=500, whole=True),
    "two_tiles_whole": dict(seqs=[(256, 1500)], hq=1, hk=1, dim=128, page=16, dtype=BF16, window=600, whole=True),
    "copied_rows_step_whole": dict(seqs=[(1, 1400), (2, 1300)], hq=4, hk=1, dim=128, page=12, dtype=BF16, window=590, whole=True),
    "heads_of_256": dict(seqs=[(3, 300)], hq=2, hk=1, dim=256, page=16, dtype=BF16, window=50),
}


@pytest.mark.parametrize("level", [-100.0, -130.0, -300.0])
@pytest.mark.parametrize("name", LOW)
def test_windows_of_very_low_scores(name, level):
    c = LOW[name]
    rng = np.random.default_rng(5)
    hq, hk, dim, page, dtype = c["hq"], c["hk"], c["dim"], c["page"], c["dtype"]
    k, v, cu, kv, table = make_cache(rng, c["seqs"], hk, dim, page, dtype, "thd", fill=float("nan"))
    # q and k point away from each other: scores of `level`, with a spread of about one
    a = (-level * dim ** -0.5) ** 0.5
    for b, (_, n) in enumerate(c["seqs"]):
        for j0 in range(0, n, page):
            m = min(page, n - j0)
            pg = int(table[b, j0 // page])
            k[pg, :m] = torch.from_numpy((-a + rng.standard_normal((m, hk, dim)) / a).astype(np.float32)).to(dtype).cuda()
            v[pg, :m] = torch.from_numpy(rng.standard_normal((m, hk, dim)).astype(np.float32)).to(dtype).cuda()
    q = torch.from_numpy((a + 0.1 * rng.standard_normal((int(cu[-1]), hq, dim))).astype(np.float32)).to(dtype).cuda()
    compare(q, k, v, cu, kv, table, max(x for x, _ in c["seqs"]), 1 if c.get("whole") else max(x for _, x in c["seqs"]), c.get("causal", True), c["window"])


@pytest.mark.parametrize("digits", [16, 23.4, 24.6, 26])
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("new,hq,dim,page,keys", [(1, 4, 128, 16, 131072), (1, 4, 64, 16, 131072), (9, 4, 64, 16, 65536), (26, 1, 128, 16, 65536),
                                                  (1, 2, 128, 12, 65532)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_dominant_key_above_a_long_tail(dtype, new, hq, dim, page, keys, first, digits):
    """One key with a score 2^digits above all others, whose values have a mean of 1: together they count."""
    if new > 1 and dtype == BF16:
        pytest.skip("one form is enough for the type with the wide exponent")
    rng = np.random.default_rng(11)
    k, v, cu, kv, table = make_cache(rng, [(new, keys)], 1, dim, page, dtype, "thd")
    at = 0 if first else keys - 200                               # (every new token sees it)
    top = (digits * np.log(2.0) * dim ** 0.5) ** 0.5
    k[int(table[0, at // page]), at % page, 0, 0] = top
    v.copy_(torch.from_numpy((1 + 0.25 * rng.standard_normal(v.shape)).astype(np.float32)))
    v[int(table[0, at // page]), at % page] = torch.from_numpy(rng.standard_normal((1, dim)).astype(np.float32)).to(dtype).cuda()
    q = torch.zeros(new, hq, dim, dtype=dtype, device="cuda")
    q[..., 0] = top
    compare(q, k, v, cu, kv, table, new, 1)                       # (one CTA: a part of its own would have a reference of its own)
