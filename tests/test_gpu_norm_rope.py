"""Norms and rotation of queries and keys, their backward pass, and the writes to a paged cache, against the FP64
definitions.  Tolerances: u |y| for the one rounding to the output type (u = half a unit in the last place of 1: 2^-11 FP16, 2^-8
BF16, 2^-24 FP32; half of the smallest subnormal for FP16) plus 32 FP32 roundings of the magnitudes that enter (the sum of squares adds 8 products
per lane and 3 to 5 shuffle levels, rsqrt 2 units, weight and rotation 5 operations); a weight gradient adds up to 256 terms in
a chain here."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as O
from paper_2609_19758_b200 import attention as A
from paper_2609_19758_b200 import build as B
from paper_2609_19758_b200 import fpsk

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
UNIT = {t: torch.finfo(t).eps / 2 for t in (F32, F16, BF16)}
TINY = {F32: 0.0, F16: 2.0 ** -25, BF16: 0.0}
E32 = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def close(got, want, tol):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.abs(got - want)[bad][:5], np.broadcast_to(tol, got.shape)[bad][:5])


def projection(rng, tokens, heads, dim, dtype, pad=0):
    """`heads` tensors (tokens, h, dim) as views into one matrix, as the columns of a projection."""
    cols = sum(heads) * dim + pad
    c = torch.from_numpy(rng.standard_normal((max(tokens, 1), cols)).astype(np.float32)).to(dtype).cuda()[:tokens]
    out, at = [], 0
    for h in heads:
        out.append(c[:, at:at + h * dim].unflatten(1, (h, dim)) if tokens else c.new_empty(0, h, dim))
        at += h * dim
    return out


def tables(n_pos, rot):
    cos, sin = A.rotary_tables(n_pos, rot)
    return cos, sin, cos.double().cpu().numpy(), sin.double().cpu().numpy()


CASES = [  # tokens, query heads, key heads, dim, rot, interleaved, in, out, padding of the rows
    (1, 4, 1, 128, 128, False, F32, BF16, 0),
    (7, 3, 2, 64, 64, False, F32, F16, 0),
    (33, 5, 1, 128, 64, True, F32, BF16, 4),
    (10, 2, 2, 96, 32, True, BF16, BF16, 0),
    (9, 2, 1, 80, 40, False, F16, F16, 0),
    (5, 1, 1, 256, 256, False, F32, BF16, 0),
    (6, 2, 1, 8, 8, False, F32, F32, 0),
    (4, 2, 3, 24, 0, False, BF16, F32, 0),
    (3, 2, 2, 64, 64, False, F32, F16, 3),      # rows at odd strides: single-element loads
    (3, 2, 2, 64, 64, True, BF16, BF16, 1),
    (2, 0, 4, 128, 128, False, F32, BF16, 0),   # keys alone
    (310, 40, 8, 128, 128, False, F32, BF16, 0),  # enough heads for four per thread
    (0, 4, 1, 128, 128, False, F32, BF16, 0),
]


@pytest.mark.parametrize("case", CASES, ids=str)
@pytest.mark.parametrize("wtype", [F32, BF16, None], ids=str)
def test_norm_rope(case, wtype):
    tokens, hq, hk, dim, rot, inter, xin, yout, pad = case
    if tokens > 100 and wtype != F32:
        pytest.skip("the large case once")
    rng = np.random.default_rng(dim + tokens)
    q, k = projection(rng, tokens, (hq, hk), dim, xin, pad)
    cos, sin, c64, s64 = tables(500, rot)
    pos = torch.from_numpy(rng.integers(0, 500, tokens).astype(np.int32)).cuda()
    w = [torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).to(wtype).cuda() if wtype else None for _ in range(2)]
    qo, ko = (torch.full((tokens, h, dim), 7.0, dtype=yout, device="cuda") for h in (hq, hk))
    args = (q if hq else None, k, cos, sin, pos, qo if hq else None, ko, w[0] if hq else None, w[1])
    A.qk_norm_rope(*args, eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    for x, y, wt in ((q, qo, w[0]), (k, ko, w[1])):
        w64 = wt.double().cpu().numpy() if wt is not None else None
        want, mag = O.norm_rope(x.double().cpu().numpy(), w64, c64[p], s64[p], rot, 1e-5, inter)
        close(y, want, UNIT[yout] * np.abs(want) + TINY[yout] + 32 * E32 * mag)
    if tokens and wtype is None and rot == 0 and xin == yout:
        assert torch.equal(qo, q)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] < 100], ids=str)
@pytest.mark.parametrize("wtype", [F32, BF16, None], ids=str)
def test_norm_rope_backward(case, wtype):
    tokens, hq, hk, dim, rot, inter, xin, gtype, pad = case
    rng = np.random.default_rng(dim + tokens + 1)
    q, k = projection(rng, tokens, (hq, hk), dim, xin, pad)
    gq, gk = projection(rng, tokens, (hq, hk), dim, gtype, pad)
    cos, sin, c64, s64 = tables(500, rot)
    pos = torch.from_numpy(rng.integers(0, 500, tokens).astype(np.int32)).cuda()
    w = [torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).to(wtype).cuda() if wtype else None for _ in range(2)]
    dq, dk = (torch.full((tokens, h, dim), 7.0, dtype=gtype, device="cuda") for h in (hq, hk))
    dw = [torch.full((dim,), 7.0, device="cuda") for _ in range(2)]
    ws = A.norm_rope_workspace(dim)
    for _ in range(2):                           # the second call finds the workspace as the first left it
        A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, dq, dk, dw[0], dw[1], ws, w[0], w[1], eps=1e-5, interleaved=inter)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    for x, g, dx, wt, dwt in ((q, gq, dq, w[0], dw[0]), (k, gk, dk, w[1], dw[1])):
        w64 = wt.double().cpu().numpy() if wt is not None else None
        want, mag, want_w, mag_w = O.norm_rope_grad(x.double().cpu().numpy(), w64, g.double().cpu().numpy(), c64[p], s64[p], rot, 1e-5, inter)
        close(dx, want, UNIT[gtype] * np.abs(want) + TINY[gtype] + 64 * E32 * mag)
        if wt is not None:
            close(dwt, want_w, (256 + 32) * E32 * mag_w)
        else:
            assert bool((dwt == 7.0).all())      # no weight, no gradient written


RING = [  # enough tokens for the ring of copied rows: tokens, query heads, key heads, dim, rot, interleaved, in, out
    (4000, 3, 2, 128, 128, False, F32, BF16),
    (15000, 2, 1, 64, 32, True, BF16, BF16),
    (3001, 30, 2, 96, 96, False, F16, F16),
    (2500, 5, 3, 256, 256, False, F32, F32),
    (20011, 1, 1, 80, 40, True, F32, F16),
]


def _plain(x, w, c, s, rot, inter, eps):
    """The forward pass in 64 bits with torch, for sizes that the loops of the definition are too slow for."""
    x = x.double()
    z = x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w.double()
    ia = torch.arange(0, rot, 2, device=x.device) if inter else torch.arange(rot // 2, device=x.device)
    ib = ia + 1 if inter else ia + rot // 2
    y = z.clone()
    y[..., ia] = z[..., ia] * c[:, None] - z[..., ib] * s[:, None]
    y[..., ib] = z[..., ib] * c[:, None] + z[..., ia] * s[:, None]
    mag = z.abs()
    mag[..., ia] = mag[..., ib] = z[..., ia].abs() + z[..., ib].abs()
    return y, mag


@pytest.mark.parametrize("case", RING, ids=str)
def test_many_tokens_forward_and_backward(case):
    tokens, hq, hk, dim, rot, inter, xin, yout = case
    rng = np.random.default_rng(tokens)
    q, k = projection(rng, tokens, (hq, hk), dim, xin)
    gq, gk = projection(rng, tokens, (hq, hk), dim, yout)
    cos, sin, _, _ = tables(300, rot)
    pos = torch.from_numpy(rng.integers(0, 300, tokens).astype(np.int32)).cuda()
    c, s = cos[pos.long()].double(), sin[pos.long()].double()
    w = [torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda(), None]
    outs = [torch.full((tokens, h, dim), 7.0, dtype=yout, device="cuda") for h in (hq, hk)]
    A.qk_norm_rope(q, k, cos, sin, pos, *outs, w[0], w[1], eps=1e-5, interleaved=inter)
    grads = [torch.full((tokens, h, dim), 7.0, dtype=yout, device="cuda") for h in (hq, hk)]
    dw = torch.full((dim,), 7.0, device="cuda")
    ws = A.norm_rope_workspace(dim)
    A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, *grads, dw, None, ws, w[0], None, eps=1e-5, interleaved=inter)
    first = [g.clone() for g in grads] + [dw.clone()]
    A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, *grads, dw, None, ws, w[0], None, eps=1e-5, interleaved=inter)
    assert all(torch.equal(a, b) for a, b in zip(first, grads + [dw]))       # the same bits again
    for x, y, g, dx, wt in ((q, outs[0], gq, grads[0], w[0]), (k, outs[1], gk, grads[1], w[1])):
        want, mag = _plain(x, wt, c, s, rot, inter, 1e-5)
        assert bool(((y.double() - want).abs() <= UNIT[yout] * want.abs() + TINY[yout] + 32 * E32 * mag).all())
        u, um = _plain(g, None, c, -s, rot, inter, 0.0)
        if wt is None:
            assert bool(((dx.double() - u).abs() <= UNIT[yout] * u.abs() + TINY[yout] + 64 * E32 * um).all())
            continue
        xd = x.double()
        r = torch.rsqrt(xd.square().mean(-1, keepdim=True) + 1e-5)
        n, gw = xd * r, u * wt.double()
        want = r * (gw - n * (gw * n).mean(-1, keepdim=True))
        mag = r * (um * wt.double().abs() + n.abs() * (um * wt.double().abs() * n.abs()).mean(-1, keepdim=True))
        assert bool(((dx.double() - want).abs() <= UNIT[yout] * want.abs() + TINY[yout] + 64 * E32 * mag).all())
        # chains of at most tokens * heads / (148 * 16) + 32 + 148 + 17 additions, and 32 roundings of a term
        chain = tokens * hq / (148 * 16) + 32 + 148 + 17 + 32
        assert bool(((dw.double() - (u * n).sum((0, 1))).abs() <= chain * E32 * (um * n.abs()).sum((0, 1))).all())


@pytest.mark.parametrize("dim,page,dtype,rot", [(128, 16, BF16, 128), (64, 5, F16, 32), (96, 24, BF16, 0)])
def test_append_of_many_tokens_equals_the_same_tokens_a_few_at_a_time(dim, page, dtype, rot):
    rng = np.random.default_rng(dim)
    seqs = [(900, 1500), (0, 7), (1, 1), (2200, 2200), (130, 100), (769, 800)]      # the fifth: 30 tokens without a place
    hq, hk = 3, 2
    kc, vc, cu, kv, table = make_cache(rng, seqs, hk, dim, page, dtype, "thd", fill=3.0)
    n = int(cu[-1])
    q, k, v = projection(rng, n, (hq, hk, hk), dim, F32)
    cos, sin, _, _ = tables(3000, rot)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda()
    whole = [torch.full((n, hq, dim), 7.0, dtype=dtype, device="cuda"), kc.clone(), vc.clone()]
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_append(A.PagedCache(whole[1], whole[2]), k, v, *dev, cos, sin, w, q=q, q_out=whole[0], q_weight=w, status=status)
    few = [torch.full((n, hq, dim), 7.0, dtype=dtype, device="cuda"), kc.clone(), vc.clone()]
    cache = A.PagedCache(few[1], few[2])
    for b, (new, keys) in enumerate(seqs):
        for t in range(0, new, 97):
            m = min(97, new - t)
            lo = int(cu[b]) + t
            at = torch.tensor([0, m], dtype=torch.int32, device="cuda")
            length = torch.tensor([keys - new + t + m], dtype=torch.int32, device="cuda")
            A.paged_append(cache, k[lo:lo + m], v[lo:lo + m], at, length, dev[2][b:b + 1], cos, sin, w, q=q[lo:lo + m], q_out=few[0][lo:lo + m],
                           q_weight=w, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert all(torch.equal(a, b) for a, b in zip(whole, few))


def test_backward_repeats_bit_for_bit_over_many_blocks():
    rng = np.random.default_rng(5)
    q, k = projection(rng, 3000, (6, 2), 128, F32)
    gq, gk = projection(rng, 3000, (6, 2), 128, BF16)
    cos, sin, _, _ = tables(64, 128)
    pos = torch.arange(3000, dtype=torch.int32, device="cuda") % 64
    w = torch.ones(128, device="cuda")
    ws = A.norm_rope_workspace(128)
    runs = []
    for _ in range(2):
        out = [torch.empty_like(gq.contiguous()), torch.empty_like(gk.contiguous()), torch.empty(128, device="cuda"), torch.empty(128, device="cuda")]
        A.qk_norm_rope_backward(q, k, gq, gk, cos, sin, pos, *out, ws, w, w)
        runs.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    n = q.double() * torch.rsqrt(q.double().square().mean(-1, keepdim=True) + 1e-6)
    # undo the rotation by autograd of the plain form
    x = q.double().detach()
    wd = w.double().clone().requires_grad_()
    c, s = cos[pos.long()].double()[:, None], sin[pos.long()].double()[:, None]
    z = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * wd
    y = torch.cat([z[..., :64] * c - z[..., 64:] * s, z[..., 64:] * c + z[..., :64] * s], -1)
    y.backward(gq.double())
    # 18000 terms in chains of at most 18000 / 592 + 592 additions
    tol = 700 * E32 * float((gq.double().abs().sum((0, 1)) * n.abs().amax()).max())
    assert float((runs[0][2].double() - wd.grad).abs().max()) <= tol


def test_autograd_function_equals_differences_of_the_definition():
    rng = np.random.default_rng(3)
    q, k = (t.contiguous().requires_grad_() for t in projection(rng, 5, (2, 1), 32, F32))
    w = torch.from_numpy((1 + 0.2 * rng.standard_normal(32)).astype(np.float32)).cuda().requires_grad_()
    cos, sin, c64, s64 = tables(50, 32)
    pos = torch.tensor([0, 49, 7, 7, 3], dtype=torch.int32, device="cuda")
    gq, gk = (torch.from_numpy(rng.standard_normal(t.shape).astype(np.float32)).cuda() for t in (q, k))
    qo, ko = A.QKNormRope.apply(q, k, w, w, cos, sin, pos, F32, 1e-5, False)
    ((qo * gq).sum() + (ko * gk).sum()).backward()
    p = pos.cpu().numpy()
    w64, h = w.detach().double().cpu().numpy(), 1e-5

    def f(q64, k64, w_):
        return sum(float(np.sum(g.double().cpu().numpy() * O.norm_rope(x, w_, c64[p], s64[p], 32, 1e-5)[0])) for x, g in ((q64, gq), (k64, gk)))

    q64, k64 = q.detach().double().cpu().numpy(), k.detach().double().cpu().numpy()
    for i in (0, 5, 31):
        d = np.zeros(32)
        d[i] = h
        assert abs((f(q64, k64, w64 + d) - f(q64, k64, w64 - d)) / (2 * h) - float(w.grad[i])) < 1e-4
    for idx in ((0, 0, 0), (4, 1, 31), (2, 0, 17)):
        d = np.zeros_like(q64)
        d[idx] = h
        assert abs((f(q64 + d, k64, w64) - f(q64 - d, k64, w64)) / (2 * h) - float(q.grad[idx])) < 1e-4


def test_positions_outside_the_tables_give_nan_and_a_status():
    q = torch.ones(4, 2, 16, device="cuda")
    cos, sin, _, _ = tables(10, 16)
    out = torch.zeros(4, 2, 16, dtype=F16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pos = torch.tensor([3, -1, 10, 9], dtype=torch.int32, device="cuda")
    A.qk_norm_rope(q, None, cos, sin, pos, out, None, status=status)
    bad = out.isnan().all(-1).all(-1)
    assert bad.tolist() == [False, True, True, False] and not out[[0, 3]].isnan().any()
    assert int(status) == fpsk.ERR_PARAM


def test_refusals():
    q = torch.ones(4, 2, 16, device="cuda")
    cos, sin, _, _ = tables(10, 16)
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    out = torch.zeros(4, 2, 16, dtype=F16, device="cuda")
    with pytest.raises(ValueError):
        A.qk_norm_rope(q, None, cos, sin, pos[:3], out, None)
    with pytest.raises(ValueError):
        A.qk_norm_rope(q, None, cos, sin, pos.long(), out, None)
    with pytest.raises(ValueError):
        A.qk_norm_rope(q, None, cos, sin, pos, out[:3], None)
    with pytest.raises(TypeError):
        A.qk_norm_rope(q.double(), None, cos, sin, pos, out, None)
    with pytest.raises(fpsk.FpskError) as e:
        A.qk_norm_rope(q, None, cos, sin, None, out, None)
    assert e.value.status == fpsk.ERR_NULL
    c12 = cos[:, :6].contiguous()
    with pytest.raises(fpsk.FpskError) as e:
        A.qk_norm_rope(q, None, c12, c12, pos, out, None)
    assert e.value.status == fpsk.ERR_PARAM      # rot_dim 12
    with pytest.raises(fpsk.FpskError) as e:
        A.qk_norm_rope(torch.ones(4, 2, 12, device="cuda"), None, None, None, None, torch.zeros(4, 2, 12, dtype=F16, device="cuda"), None)
    assert e.value.status == fpsk.ERR_SHAPE
    with pytest.raises(fpsk.FpskError) as e:
        A.qk_norm_rope(q, None, cos, sin, pos, out, None, eps=-1.0)
    assert e.value.status == fpsk.ERR_PARAM
    with pytest.raises(fpsk.FpskError) as e:
        A.qk_norm_rope_backward(q, None, out, None, cos, sin, pos, out, None, None, None, torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == fpsk.ERR_WORKSPACE


# ---------------------------------------------------------------- appending
APPENDS = [  # (new, keys) per sequence, query heads, key heads, dim, rot, page, in, cache type, order, interleaved
    ([(1, 1)], 4, 1, 128, 128, 16, F32, BF16, "thd", False),
    ([(3, 17), (1, 16), (0, 5), (9, 9), (0, 0), (2, 40)], 6, 2, 64, 64, 8, F32, F16, "thd", False),
    ([(5, 33), (4, 3)], 2, 2, 128, 64, 16, BF16, BF16, "htd", True),   # the second: a token without a place
    ([(7, 100)], 0, 3, 96, 96, 5, F32, BF16, "htd", False),            # pages of an odd size, no queries
    ([(40, 700), (1, 3)], 8, 8, 80, 40, 24, F16, F16, "thd", False),
    ([(1, 1 + 13 * i) for i in range(70)], 4, 2, 256, 0, 16, F32, BF16, "thd", False),
    ([(0, 0)] * 300 + [(2, 5)] + [(0, 3)] * 40 + [(1, 1)], 4, 2, 64, 64, 16, F32, BF16, "thd", False),
]


def make_cache(rng, seqs, hk, dim, page, dtype, order, extra=2, fill=0.0):
    n = [-(-kv // page) for _, kv in seqs]
    total = sum(n) + extra
    shape = (total, page, hk, dim) if order == "thd" else (total, hk, page, dim)
    made = [torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(2)]
    k, v = made if order == "thd" else [t.permute(0, 2, 1, 3) for t in made]
    perm = rng.permutation(total)
    table = np.full((len(seqs), max(n + [0]) + 1), -1, dtype=np.int32)
    at = 0
    for b, c in enumerate(n):
        table[b, :c] = perm[at:at + c]
        at += c
    cu = np.concatenate([[0], np.cumsum([a for a, _ in seqs])]).astype(np.int32)
    kv = np.array([b for _, b in seqs], dtype=np.int32)
    return k, v, cu, kv, table


@pytest.mark.parametrize("case", APPENDS, ids=lambda c: str(c)[:60])
@pytest.mark.parametrize("normed", [True, False])
def test_append(case, normed):
    seqs, hq, hk, dim, rot, page, xin, ctype, order, inter = case
    rng = np.random.default_rng(dim + page)
    kc, vc, cu, kv, table = make_cache(rng, seqs, hk, dim, page, ctype, order, fill=3.0)
    n = int(cu[-1])
    q, k, v = projection(rng, n, (hq, hk, hk), dim, xin)
    cos, sin, c64, s64 = tables(1000, rot)
    w = [torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).cuda() if normed else None for _ in range(2)]
    qo = torch.full((n, hq, dim), 7.0, dtype=ctype, device="cuda")
    cache = A.PagedCache(kc, vc)
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_append(cache, k, v, *dev, cos, sin, w[1], q=q if hq else None, q_out=qo if hq else None, q_weight=w[0] if hq else None,
                   eps=1e-5, interleaved=inter, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    at = O.places(cu, kv, page, table)
    pos = np.array([max(p, 0) for _, p, _, _ in at])
    there = np.array([p >= 0 for _, p, _, _ in at])
    w64 = [x.double().cpu().numpy() if x is not None else None for x in w]
    want_k, mag = O.norm_rope(k.double().cpu().numpy(), w64[1], c64[pos], s64[pos], rot, 1e-5, inter)
    tol_k = UNIT[ctype] * np.abs(want_k) + TINY[ctype] + 32 * E32 * mag
    k_all, v_all = kc.double().cpu().numpy(), vc.double().cpu().numpy()
    seen = np.zeros(k_all.shape[:2], dtype=bool)
    for t, (_, p, pg, row) in enumerate(at):
        if p < 0:
            continue
        seen[pg, row] = True
        assert np.all(np.abs(k_all[pg, row] - want_k[t]) <= tol_k[t])
        assert np.array_equal(v_all[pg, row], v[t].to(ctype).double().cpu().numpy())
    assert np.all(k_all[~seen] == 3.0) and np.all(v_all[~seen] == 3.0)      # nothing else is touched
    if hq:
        want_q, mag = O.norm_rope(q.double().cpu().numpy(), w64[0], c64[pos], s64[pos], rot, 1e-5, inter)
        if rot:
            want_q[~there], mag[~there] = 0.0, 0.0
        close(qo, want_q, UNIT[ctype] * np.abs(want_q) + TINY[ctype] + 32 * E32 * mag)


def test_append_reports_pages_outside_the_cache_and_writes_the_others():
    rng = np.random.default_rng(0)
    kc, vc, cu, kv, table = make_cache(rng, [(20, 40)], 1, 64, 16, BF16, "thd")
    table[0, 1] = 1000
    _, k, v = projection(rng, 20, (0, 1, 1), 64, F32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    A.paged_append(A.PagedCache(kc, vc), k, v, *(torch.from_numpy(x).cuda() for x in (cu, kv, table)), status=status)
    assert int(status) == fpsk.ERR_PARAM
    assert torch.equal(vc[int(table[0, 2]), :8, 0], v[12:, 0].to(BF16))


def test_append_with_given_positions_on_another_stream():
    rng = np.random.default_rng(4)
    kc, vc, cu, kv, table = make_cache(rng, [(3, 9), (2, 2)], 2, 64, 16, F16, "thd")
    _, k, v = projection(rng, 5, (0, 2, 2), 64, F32)
    cos, sin, c64, s64 = tables(300, 64)
    pos = torch.tensor([299, 0, 17, 5, 100], dtype=torch.int32, device="cuda")
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    A.paged_append(A.PagedCache(kc, vc), k, v, *dev, cos, sin, positions=pos, stream=st)
    st.synchronize()
    p = pos.cpu().numpy()
    want, mag = O.norm_rope(k.double().cpu().numpy(), None, c64[p], s64[p], 64, 1e-6)
    for t, (_, _, pg, row) in enumerate(O.places(cu, kv, 16, table)):
        assert np.all(np.abs(kc[pg, row].double().cpu().numpy() - want[t]) <= UNIT[F16] * np.abs(want[t]) + TINY[F16] + 32 * E32 * mag[t])


def test_append_refusals():
    rng = np.random.default_rng(0)
    kc, vc, cu, kv, table = make_cache(rng, [(2, 4)], 1, 64, 16, BF16, "thd")
    _, k, v = projection(rng, 2, (0, 1, 1), 64, F32)
    dev = [torch.from_numpy(x).cuda() for x in (cu, kv, table)]
    with pytest.raises(ValueError):
        A.PagedCache(kc.float(), vc.float())
    with pytest.raises(ValueError):
        A.PagedCache(kc, vc[1:])
    with pytest.raises(ValueError):
        A.paged_append(A.PagedCache(kc, vc), k[..., :32], v[..., :32], *dev)
    with pytest.raises(ValueError):
        A.paged_append(A.PagedCache(kc, vc), k, v, dev[0].long(), dev[1], dev[2])
    with pytest.raises(ValueError):
        A.paged_append(A.PagedCache(kc, vc), k, v, dev[0], dev[1], dev[2][:0])
