"""The attention operators beside a verified projection: what is measured, and their plain forms.

A transformer layer's QKV projection is a GEMM whose FP32 accumulator is delivered un-narrowed, so that it can be
verified.  The operators here take it from there: they read the accumulator (or a 16-bit tensor) and do what an
attention layer does before its output projection.

  norm_rope        y = R_pos (x rsqrt(mean(x^2) + eps) * w) for every query and key head; rounded once
  norm_rope_grad   its backward pass: gradients of the inputs and of both weights
  append           keys (normed, rotated) and values written to the pages of a cache, queries normed and rotated beside them
  attention        a chunk of new tokens (one or many) of every sequence over its pages

With `own` false, `run` computes them with elementary torch operations in 32 bits, rounded once at the end; with `own`
true it calls the library's entry points.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------- cases
def _norm(name, op, tokens, hq, hk, dim, rot, src, dst, interleaved=False):
    return {"name": name, "op": op, "tokens": tokens, "hq": hq, "hk": hk, "dim": dim, "rot": rot, "src": src, "dst": dst,
            "interleaved": interleaved}


def _append(name, seqs, new, ctx, hq, hk, dim, rot, page, src, dst, norm, ragged, mix):
    return {"name": name, "op": "append", "seqs": seqs, "new": new, "ctx": ctx, "hq": hq, "hk": hk, "dim": dim, "rot": rot,
            "page": page, "src": src, "dst": dst, "norm": norm, "ragged": ragged, "mix": mix}


def _attention(name, seqs, new, ctx, hq, hk, dim, page, dst, window, ragged, mix, causal=True):
    return {"name": name, "op": "attention", "seqs": seqs, "new": new, "ctx": ctx, "hq": hq, "hk": hk, "dim": dim, "page": page,
            "dst": dst, "window": window, "ragged": ragged, "mix": mix, "causal": causal}


def listed():
    return [
        # one token of one request, 32 query and 8 key heads: the smallest call, all latency
        _norm("norm_rope_step", "norm_rope", 1, 32, 8, 128, 128, "f32", "bf16"),
        # a prompt of 4096 tokens, 32 heads of 128 (the 4096 x 4096 Q and K projections of the transformer shape set)
        _norm("norm_rope_prompt", "norm_rope", 4096, 32, 32, 128, 128, "f32", "f16"),
        # the same tokens in training: gradients of the projection's output and of the two weights
        _norm("norm_rope_grad", "norm_rope_grad", 4096, 32, 32, 128, 128, "f32", "bf16"),
        # an odd micro-batch of a narrow model: 16-bit input, part of the head rotated, pairs side by side
        _norm("norm_rope_grad_odd", "norm_rope_grad", 1021, 28, 4, 96, 32, "bf16", "bf16", True),
        # one decoding step of 64 requests: queries rotated, keys and values to their pages
        _append("append_step", 64, 1, 4000, 32, 8, 128, 128, 16, "f32", "bf16", True, True, 1),
        # the prompts of a dozen requests at once, of uneven lengths
        _append("append_prompts", 12, 1500, 700, 32, 32, 128, 128, 64, "f32", "f16", False, True, 2),
        # one decoding step of one request with a short context: latency
        _attention("attention_step", 1, 1, 1000, 32, 8, 128, 16, "bf16", -1, False, 3),
        # one decoding step of 96 requests of uneven context, up to 8192
        _attention("attention_batch", 96, 1, 8191, 32, 8, 128, 16, "bf16", -1, True, 4),
        # four drafted tokens of one request over a quarter million tokens, 64 query heads: long axis, few rows
        _attention("attention_long", 1, 4, 262140, 64, 8, 128, 64, "bf16", -1, False, 5),
        # chunks of some requests (a few hundred new tokens each, uneven), 32 heads without sharing
        _attention("attention_chunks", 6, 500, 7000, 32, 32, 128, 16, "f16", -1, True, 6),
        # a chunk of 4096 tokens of one long prompt: the largest, bound by the tensor cores
        _attention("attention_prompt", 1, 4096, 12288, 32, 8, 128, 128, "bf16", -1, False, 7),
        # a narrow model with a sliding window, 7 query heads to a key head, pages of 24
        _attention("attention_window", 5, 700, 5000, 14, 2, 64, 24, "f16", 1000, True, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(rng):
    op = rng.choice(["norm_rope", "norm_rope_grad", "append", "attention", "attention", "attention"])
    dim = rng.choice([64, 128, 128, 96, 80])
    hk = rng.choice([1, 2, 4, 8, 8, 16, 32])
    group = rng.choice([1, 1, 2, 4, 4, 7, 8])
    dst = rng.choice(["bf16", "f16"])
    if op in ("norm_rope", "norm_rope_grad"):
        rot = rng.choice([dim, dim, dim // 16 * 8])
        return {"op": op, "tokens": _log(rng, 1, 8192), "hq": hk * group, "hk": hk, "dim": dim, "rot": rot,
                "src": rng.choice(["f32", "f32", dst]), "dst": dst, "interleaved": rng.random() < 0.3}
    page = rng.choice([16, 16, 32, 64, 128, 24, 8])
    mix = rng.randrange(1 << 20)
    if op == "append":
        return {"op": op, "seqs": _log(rng, 1, 128), "new": rng.choice([1, 1, _log(rng, 2, 2048)]), "ctx": _log(rng, 1, 4000),
                "hq": hk * group, "hk": hk, "dim": dim, "rot": rng.choice([dim, dim, dim // 16 * 8]), "page": page,
                "src": rng.choice(["f32", "f32", dst]), "dst": dst, "norm": rng.random() < 0.5, "ragged": rng.random() < 0.7,
                "mix": mix}
    return {"op": op, "seqs": _log(rng, 1, 128), "new": rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 4096)]),
            "ctx": _log(rng, 1, 131072), "hq": hk * group, "hk": hk, "dim": dim, "page": page, "dst": dst,
            "window": rng.choice([-1, -1, -1, _log(rng, 16, 4096)]), "ragged": rng.random() < 0.7, "mix": mix,
            "causal": rng.random() < 0.85}


def draw(rng):
    """One more case of the ranges above; no dearer than the largest listed one, in work or in what the plain form holds."""
    while True:
        c = _drawn(rng)
        if c["op"] in ("norm_rope", "norm_rope_grad"):
            if c["tokens"] * (c["hq"] + c["hk"]) * c["dim"] <= 4096 * 64 * 128:
                return c
            continue
        q, kv = lengths(c)
        if c["seqs"] * (c["ctx"] + c["new"] + c["page"]) * c["hk"] * c["dim"] > 262144 * 8 * 128:
            continue
        if sum(q) * (c["hq"] + 2 * c["hk"]) * c["dim"] > 18000 * 96 * 128:
            continue
        if c["op"] == "attention" and c["seqs"] * max(q) * c["hq"] * max(kv) > 4096 * 32 * 16384:
            continue
        return c


def lengths(case):
    """New tokens and keys (the new ones among them) of every sequence."""
    n, new, ctx = case["seqs"], case["new"], case["ctx"]
    if not case["ragged"]:
        return [new] * n, [ctx + new] * n
    r = random.Random(case["mix"])
    q = [new if new == 1 else (0 if r.random() < 0.06 else r.randint(1, new)) for _ in range(n)]
    kv = [int(math.exp(r.uniform(0.0, math.log(ctx + 1)))) - 1 for _ in range(n)]
    at = r.randrange(n)
    q[at], kv[at] = new, ctx
    return q, [a + b for a, b in zip(q, kv)]


def pages(case):
    _, kv = lengths(case)
    return [-(-k // case["page"]) for k in kv]


def work(case):
    if case["op"] in ("norm_rope", "norm_rope_grad"):
        n = case["tokens"] * (case["hq"] + case["hk"]) * case["dim"]
        table = case["tokens"] * (case["rot"] * 4 + 4)
        if case["op"] == "norm_rope":
            return {"bytes": n * (SIZE[case["src"]] + SIZE[case["dst"]]) + table + 8 * case["dim"], "flops": 8 * n}
        return {"bytes": n * (SIZE[case["src"]] + 2 * SIZE[case["dst"]]) + table + 16 * case["dim"], "flops": 20 * n}
    q, kv = lengths(case)
    if case["op"] == "append":
        n = sum(q) * (case["hq"] + 2 * case["hk"]) * case["dim"]
        return {"bytes": n * (SIZE[case["src"]] + SIZE[case["dst"]]) + sum(q) * (case["rot"] * 4 + 4), "flops": 8 * n}
    pairs, keys = 0, 0
    for a, b in zip(q, kv):
        # the key ranges of the new tokens: first and one past the last, in closed form over the sequence
        pairs += _pairs(a, b, case["window"], case["causal"])
        if a:
            first = max(0, b - a - case["window"]) if case["window"] >= 0 else 0
            keys += b - first
    size = SIZE[case["dst"]]
    return {"bytes": keys * case["hk"] * case["dim"] * 2 * size + sum(q) * case["hq"] * (case["dim"] * 2 * size + 4),
            "flops": 4 * case["dim"] * case["hq"] * pairs}


def _pairs(q, kv, window, causal):
    """Pairs of a new token at position p = kv - q + t and a key j with max(0, p - window) <= j < (p + 1 if causal else kv)."""
    upper = q * (kv - q) + q * (q + 1) // 2 if causal else q * kv
    if window < 0:
        return upper
    over = [kv - q - window, kv - 1 - window]          # keys before the window of the first and of the last token
    lo = max(0, over[0])
    return upper - (over[1] * (over[1] + 1) - lo * (lo - 1)) // 2 if over[1] > 0 else upper


# ---------------------------------------------------------------------------------------------- inputs
def _tables(n_pos, rot, device):
    """cos and sin of pos * 10000^(-2 i / rot), as FP32 tables (positions, rot / 2)."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / max(rot, 1))
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * inv
    return a.cos().float(), a.sin().float()


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _weight(g, dim):
    return 1.0 + 0.2 * _randn(g, dim)


def _accumulator(g, tokens, cols, kind):
    """The output of a projection: FP32 accumulators with channels of uneven size."""
    x = _randn(g, tokens, cols)
    x *= torch.exp(0.5 * _randn(g, cols))
    return x.to(TYPES[kind])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case)}
    dim = case["dim"]
    hq, hk = case["hq"], case["hk"]
    if case["op"] in ("norm_rope", "norm_rope_grad"):
        t = case["tokens"]
        c = _accumulator(g, t, (hq + 2 * hk) * dim, case["src"])           # Q, K and V columns of one projection
        s["q"], s["k"] = c[:, :hq * dim].view(t, hq, dim), c[:, hq * dim:(hq + hk) * dim].view(t, hk, dim)
        s["cos"], s["sin"] = _tables(16384, case["rot"], "cuda")
        s["positions"] = torch.randint(0, 16384, (t,), generator=g, device="cuda", dtype=torch.int32)
        s["q_weight"], s["k_weight"] = _weight(g, dim), _weight(g, dim)
        dst = TYPES[case["dst"]]
        s["q_out"], s["k_out"] = (torch.zeros(t, h, dim, dtype=dst, device="cuda") for h in (hq, hk))
        if case["op"] == "norm_rope_grad":
            s["dq_out"], s["dk_out"] = _randn(g, t, hq, dim).to(dst), _randn(g, t, hk, dim).to(dst)
            s["dq_weight"], s["dk_weight"] = torch.zeros(dim, device="cuda"), torch.zeros(dim, device="cuda")
        return s
    q_len, kv_len = lengths(case)
    n_pages = pages(case)
    total, page = sum(n_pages), case["page"]
    spare = 3 + total // 50
    dst = TYPES[case["dst"]]
    # cache (pages, page, key heads, dim); the pages of a sequence lie anywhere; what the table does not use is -1
    s["k_cache"] = _randn(g, total + spare, page, hk, dim).to(dst)
    s["v_cache"] = _randn(g, total + spare, page, hk, dim).to(dst)
    order = torch.randperm(total + spare, generator=g, device="cuda")
    count = torch.tensor(n_pages, device="cuda")
    col = torch.arange(max(max(n_pages), 1) + 1, device="cuda")[None, :]
    used = col < count[:, None]
    start = torch.cumsum(count, 0) - count
    s["block_table"] = torch.where(used, order[(start[:, None] + col).clamp(max=total + spare - 1)], torch.full_like(col, -1)).to(torch.int32)
    s["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    cu = [0]
    for a in q_len:
        cu.append(cu[-1] + a)
    s["cu_q"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    t = cu[-1]
    s["max_q"], s["max_kv"] = max(q_len), max(kv_len)
    if case["op"] == "append":
        c = _accumulator(g, t, (hq + 2 * hk) * dim, case["src"])
        s["q"] = c[:, :hq * dim].view(t, hq, dim)
        s["k"] = c[:, hq * dim:(hq + hk) * dim].view(t, hk, dim)
        s["v"] = c[:, (hq + hk) * dim:].view(t, hk, dim)
        s["cos"], s["sin"] = _tables(8192, case["rot"], "cuda")
        s["q_weight"], s["k_weight"] = (_weight(g, dim), _weight(g, dim)) if case["norm"] else (None, None)
        s["q_out"] = torch.zeros(t, hq, dim, dtype=dst, device="cuda")
        return s
    # what lies behind the last key of a sequence, and in pages that no sequence has, was never written: NaN here
    seen = torch.zeros((total + spare) * page, dtype=torch.bool, device="cuda")
    at = torch.arange(s["block_table"].shape[1] * page, device="cuda")[None, :].expand(case["seqs"], -1)
    seq = torch.arange(case["seqs"], device="cuda")[:, None].expand_as(at)
    live = at < s["kv_len"][:, None]
    seen[s["block_table"].long()[seq[live], at[live] // page] * page + at[live] % page] = True
    seen = seen.view(total + spare, page)
    s["k_cache"][~seen] = float("nan")
    s["v_cache"][~seen] = float("nan")
    s["q"] = (1.5 * _randn(g, t, hq, dim)).to(dst)
    s["out"] = torch.zeros(t, hq, dim, dtype=dst, device="cuda")
    s["lse"] = torch.zeros(t, hq, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- plain forms (32 bits)
def _pair_index(dim, rot, interleaved, device):
    i = torch.arange(rot // 2, device=device)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _rotate(x, c, s, rot, interleaved):
    """Pairs (a, b) of the first `rot` channels to (a c - b s, b c + a s); c and s are (tokens, rot / 2)."""
    ia, ib = _pair_index(x.shape[-1], rot, interleaved, x.device)
    a, b = x[..., ia], x[..., ib]
    y = x.clone()
    y[..., ia] = a * c[:, None, :] - b * s[:, None, :]
    y[..., ib] = b * c[:, None, :] + a * s[:, None, :]
    return y


def _plain_head(x, w, c, s, rot, interleaved):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    return _rotate(x, c, s, rot, interleaved)


def _plain_head_grad(x, w, dy, c, s, rot, interleaved):
    x = x.float()
    u = _rotate(dy.float(), c, -s, rot, interleaved)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = u * w
    return r * (dn - n * (dn * n).mean(-1, keepdim=True)), (u * n).sum((0, 1))


def _plain_norm_rope(s):
    case = s["case"]
    at = s["positions"].long()
    c, sn = s["cos"][at], s["sin"][at]
    dst = TYPES[case["dst"]]
    if case["op"] == "norm_rope":
        return {n: _plain_head(s[n], s[n + "_weight"], c, sn, case["rot"], case["interleaved"]).to(dst) for n in ("q", "k")}
    dq, dqw = _plain_head_grad(s["q"], s["q_weight"], s["dq_out"], c, sn, case["rot"], case["interleaved"])
    dk, dkw = _plain_head_grad(s["k"], s["k_weight"], s["dk_out"], c, sn, case["rot"], case["interleaved"])
    return {"dq": dq.to(dst), "dk": dk.to(dst), "dq_weight": dqw, "dk_weight": dkw}


def _token_places(s):
    """Sequence and position of every new token."""
    cu, t = s["cu_q"].long(), s["q"].shape[0]
    tok = torch.arange(t, device="cuda")
    seq = torch.searchsorted(cu[1:], tok, right=True)
    return seq, s["kv_len"].long()[seq] - cu[seq + 1] + tok


def _plain_append(s):
    case = s["case"]
    seq, pos = _token_places(s)
    slot_page = s["block_table"].long()[seq, pos // case["page"]]
    c, sn = s["cos"][pos], s["sin"][pos]
    dst = TYPES[case["dst"]]
    q = _plain_head(s["q"], s["q_weight"], c, sn, case["rot"], False).to(dst)
    s["k_cache"][slot_page, pos % case["page"]] = _plain_head(s["k"], s["k_weight"], c, sn, case["rot"], False).to(dst)
    s["v_cache"][slot_page, pos % case["page"]] = s["v"].to(dst)
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    case = s["case"]
    b, hq, hk, dim, page = case["seqs"], case["hq"], case["hk"], case["dim"], case["page"]
    nq, nk = s["max_q"], s["max_kv"]
    cu, kv_len = s["cu_q"].long(), s["kv_len"].long()
    q_len = cu[1:] - cu[:-1]
    t = torch.arange(nq, device="cuda")
    tok = (cu[:-1, None] + t).clamp(max=s["q"].shape[0] - 1)
    table = s["block_table"].long().clamp(min=0)[:, :-(-nk // page)]
    j = torch.arange(nk, device="cuda")
    dead = (j >= kv_len[:, None])[:, :, None, None]
    k = s["k_cache"][table].view(b, -1, hk, dim)[:, :nk].float().masked_fill_(dead, 0.0)
    v = s["v_cache"][table].view(b, -1, hk, dim)[:, :nk].float().masked_fill_(dead, 0.0)
    # queries of the heads that share a key head, as the rows of one product
    q = s["q"][tok].float().view(b, nq, hk, hq // hk, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dim)
    scores = (q @ k.permute(0, 2, 3, 1)).view(b, hk, hq // hk, nq, nk)
    scores *= 1.0 / math.sqrt(dim)
    pos = (kv_len - q_len)[:, None, None] + t[None, :, None]
    bad = j[None, None, :] >= kv_len[:, None, None]
    if case["causal"]:
        bad = bad | (j[None, None, :] > pos)
    if case["window"] >= 0:
        bad = bad | (j[None, None, :] < pos - case["window"])
    scores.masked_fill_(bad[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.view(b, hk, -1, nk) @ v.permute(0, 2, 1, 3)).view(b, hk, hq // hk, nq, dim) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (total.log() + top)[..., 0]
    mine = t < q_len[:, None]
    out = out.permute(0, 3, 1, 2, 4).reshape(b, nq, hq, dim)[mine]
    return {"out": out.to(TYPES[case["dst"]]), "lse": lse.permute(0, 3, 1, 2).reshape(b, nq, hq)[mine]}


# ---------------------------------------------------------------------------------------------- the library's operators
def _own_norm_rope(s):
    from paper_2609_19758_b200 import attention as A
    case = s["case"]
    if case["op"] == "norm_rope":
        A.qk_norm_rope(s["q"], s["k"], s["cos"], s["sin"], s["positions"], s["q_out"], s["k_out"], s["q_weight"], s["k_weight"],
                       eps=EPS, interleaved=case["interleaved"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if "ws" not in s:                                        # kept by a training program from step to step
        s["ws"] = A.norm_rope_workspace(case["dim"])
    A.qk_norm_rope_backward(s["q"], s["k"], s["dq_out"], s["dk_out"], s["cos"], s["sin"], s["positions"], s["q_out"], s["k_out"],
                            s["dq_weight"], s["dk_weight"], s["ws"], s["q_weight"], s["k_weight"], eps=EPS,
                            interleaved=case["interleaved"])
    return {"dq": s["q_out"], "dk": s["k_out"], "dq_weight": s["dq_weight"], "dk_weight": s["dk_weight"]}


def _own_cache(s):
    from paper_2609_19758_b200 import attention as A
    if "cache" not in s:                                     # the handle of a serving program's cache, and its workspace
        s["cache"] = A.PagedCache(s["k_cache"], s["v_cache"])
        if s["case"]["op"] == "attention":
            s["ws"] = A.attention_workspace()
    return A, s["cache"]


def _own_append(s):
    A, cache = _own_cache(s)
    A.paged_append(cache, s["k"], s["v"], s["cu_q"], s["kv_len"], s["block_table"], s["cos"], s["sin"], s["k_weight"],
                   q=s["q"], q_out=s["q_out"], q_weight=s["q_weight"], eps=EPS)
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attention(s):
    A, cache = _own_cache(s)
    case = s["case"]
    A.paged_attention(cache, s["q"], s["out"], s["cu_q"], s["kv_len"], s["block_table"], s["ws"], s["max_q"], s["max_kv"],
                      causal=case["causal"], window=case["window"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    op = state["case"]["op"]
    if op in ("norm_rope", "norm_rope_grad"):
        return _own_norm_rope(state) if own else _plain_norm_rope(state)
    if op == "append":
        return _own_append(state) if own else _plain_append(state)
    return _own_attention(state) if own else _plain_attention(state)


# ---------------------------------------------------------------------------------------------- 64 bits, from the definitions
def _exact_rotation(c, s, dim, rot, interleaved):
    """The rotation of every token as a pair of (tokens, dim) factors and the partner of each channel: y = x f + x[partner] h."""
    f = torch.ones(c.shape[0], dim, dtype=torch.float64, device=c.device)
    h = torch.zeros_like(f)
    partner = torch.arange(dim, device=c.device)
    if rot:
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
        f[:, lo], f[:, hi] = c.double(), c.double()
        h[:, lo], h[:, hi] = -s.double(), s.double()
        first = partner[lo].clone()
        partner[lo] = partner[hi].clone()
        partner[hi] = first
    return f[:, None, :], h[:, None, :], partner


def _exact_normed(x, w):
    x = x.double()
    if w is None:
        return x, None
    r = 1.0 / torch.sqrt(torch.square(x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    return x * r * w.double(), r


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, s)
    if case["op"] == "append":
        q_len, kv_len = lengths(case)
        place = [(b, kv - n + i) for b, (n, kv) in enumerate(zip(q_len, kv_len)) for i in range(n)]
        seq, pos = (torch.tensor(x, device="cuda") for x in zip(*place))
    else:
        pos = s["positions"].long()
    f, h, partner = _exact_rotation(s["cos"][pos], s["sin"][pos], case["dim"], case["rot"], case.get("interleaved", False))
    if case["op"] in ("norm_rope", "append"):
        y = {}
        for n in ("q", "k"):
            z = _exact_normed(s[n], s[n + "_weight"])[0]
            y[n] = z * f + z[..., partner] * h
        if case["op"] == "norm_rope":
            return y
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        where = s["block_table"].long()[seq, pos // case["page"]] * case["page"] + pos % case["page"]
        kc.view(-1, case["hk"], case["dim"])[where] = y["k"]
        vc.view(-1, case["hk"], case["dim"])[where] = s["v"].double()
        return {"q": y["q"], "k_cache": kc, "v_cache": vc}
    got = {}
    for n in ("q", "k"):
        x, w, dy = s[n].double(), s[n + "_weight"].double(), s["d%s_out" % n].double()
        z, r = _exact_normed(s[n], torch.ones_like(w))
        u = dy * f - dy[..., partner] * h                               # the transpose of the rotation
        got["d%s_weight" % n] = torch.einsum("thd,thd->d", u, z)
        g = u * w
        got["d" + n] = r * g - x * r ** 3 * (g * x).sum(-1, keepdim=True) / case["dim"]
    return got


def _exact_attention(case, s):
    """Sequence by sequence, key head by key head, blocks of queries."""
    if 4.0 * case["dim"] * case["hq"] * sum(a * b for a, b in zip(*lengths(case))) > 3e13:
        return None
    q_len, kv_len = lengths(case)
    group, page = case["hq"] // case["hk"], case["page"]
    out = torch.zeros(sum(q_len), case["hq"], case["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((sum(q_len), case["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, kv) in enumerate(zip(q_len, kv_len)):
        if n == 0:
            continue
        own_pages = s["block_table"][b, :-(-kv // page)].long()
        keys, values = (s[c][own_pages].reshape(-1, case["hk"], case["dim"])[:kv] for c in ("k_cache", "v_cache"))
        for t0 in range(0, n, 1024):
            t1 = min(n, t0 + 1024)
            pos = torch.arange(kv - n + t0, kv - n + t1, device="cuda")
            lo = int(pos[0]) - case["window"] if case["window"] >= 0 else 0
            lo, hi = max(0, lo), (int(pos[-1]) + 1 if case["causal"] else kv)
            if hi <= lo:
                continue
            j = torch.arange(lo, hi, device="cuda")
            allowed = torch.ones(len(pos), hi - lo, dtype=torch.bool, device="cuda")
            if case["causal"]:
                allowed &= j[None, :] <= pos[:, None]
            if case["window"] >= 0:
                allowed &= j[None, :] + case["window"] >= pos[:, None]
            for h in range(case["hk"]):
                rows = s["q"][first + t0:first + t1, h * group:(h + 1) * group].double()
                e = torch.einsum("tgd,kd->gtk", rows, keys[lo:hi, h].double()) * case["dim"] ** -0.5
                e = torch.where(allowed, e, torch.full_like(e, -math.inf))
                l = torch.logsumexp(e, -1)
                p = torch.exp(e - torch.where(torch.isinf(l), torch.zeros_like(l), l)[..., None])
                out[first + t0:first + t1, h * group:(h + 1) * group] = torch.einsum("gtk,kd->tgd", p, values[lo:hi, h].double())
                lse[first + t0:first + t1, h * group:(h + 1) * group] = l.T
        first += n
    return {"out": out, "lse": lse}
