"""The operators on the other accumulators of a verified decoder, the output projection's and the head's: what is measured, and
their plain forms.

  norm         h = x + residual (stored), y = h rsqrt(mean(h^2) + eps) w, in 16 bits, or in e4m3 with a scale for each group of channels
  norm_grad    its backward pass: the gradient of the sum, with what arrives through the residual stream, and of the weight
  logits       penalties for repeated tokens, biases and grammar masks on a head's logits; the greedy token and the log-sum-exp
  distill      the loss of logits against a teacher's top logits, with the gradient of the weighted sum in the same call
  distill_eval the loss alone
  distill_grad the loss, then the gradient for any gradients of the rows' losses, as automatic differentiation asks for them

With `own` false, `run` computes them with elementary torch operations in 32 bits, rounded once at the end; with `own` true it calls
the library's entry points.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}
EPS = 1e-6
TOP = 448.0                                             # the largest e4m3 value
LEAST_SCALE = 2.0 ** -126


# ---------------------------------------------------------------------------------------------- cases
def _norm(name, tokens, dim, src, res, dst, group=0):
    return {"name": name, "op": "norm", "tokens": tokens, "dim": dim, "src": src, "res": res, "dst": dst, "group": group}


def _norm_grad(name, tokens, dim, src, grad):
    return {"name": name, "op": "norm_grad", "tokens": tokens, "dim": dim, "src": src, "grad": grad}


def _logits(name, rows, vocab, src, dst, history, biases, mask, pick):
    return {"name": name, "op": "logits", "rows": rows, "vocab": vocab, "src": src, "dst": dst, "history": history, "biases": biases,
            "mask": mask, "pick": pick}


def _distill(name, op, rows, vocab, src, grad, top, temperature=1.0, normalize=True):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "src": src, "grad": grad, "top": top, "temperature": temperature,
            "normalize": normalize}


def listed():
    return [
        # one token between two layers of 4096 channels: all latency
        _norm("norm_step", 1, 4096, "f32", "bf16", "bf16"),
        # a prompt of 4096 tokens behind the 4096 x 4096 output projection
        _norm("norm_prompt", 4096, 4096, "f32", "bf16", "bf16"),
        # a wide model's tokens into a product in 8 bits, a scale for each 128 channels
        _norm("norm_e4m3", 8192, 8192, "f32", "bf16", "e4m3", 128),
        # training: gradients of the prompt's tokens
        _norm_grad("norm_grad", 4096, 4096, "bf16", "bf16"),
        # an odd micro-batch of an odd width (rows that start off 16 bytes), gradients in 32 bits
        _norm_grad("norm_grad_odd", 1021, 2050, "f16", "f32"),
        # one request's step: 32000 logits, a thousand tokens of history, all penalties: latency
        _logits("logits_step", 1, 32000, "f32", "f32", 1000, 0, "none", True),
        # a step of 96 requests over 131072 tokens, histories of up to 4096, a third of them held to a grammar; the tokens alone are wanted
        _logits("logits_batch", 96, 131072, "f32", "none", 4096, 64, "some", True),
        # drafted positions of many requests in an odd vocabulary, narrow logits adjusted to FP32
        _logits("logits_drafts", 640, 50257, "bf16", "f32", 700, 16, "all", False),
        # a few positions: latency of a long axis
        _distill("distill_small", "distill", 5, 131072, "f32", "bf16", 32),
        # the validation set: losses alone
        _distill("distill_eval", "distill_eval", 2048, 65536, "bf16", "none", 64, 2.0),
        # a training step of 4096 positions over 131072 tokens: the largest
        _distill("distill_step", "distill", 4096, 131072, "f32", "bf16", 64, 1.0, False),
        # losses whose gradients come later, odd vocabulary, a fifth of the positions padding
        _distill("distill_grad_odd", "distill_grad", 1500, 50257, "f16", "f16", 100, 1.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above; no dearer than the largest listed one."""
    op = rng.choice(["norm", "norm_grad", "logits", "logits", "distill", "distill_eval", "distill_grad"])
    half = rng.choice(["bf16", "f16"])
    src = rng.choice(["f32", half])
    if op in ("norm", "norm_grad"):
        dim = rng.choice([_log(rng, 64, 16384), 8 * _log(rng, 8, 2048), 256 * rng.randint(1, 64)])
        tokens = _log(rng, 1, min(16384, (1 << 26) // dim))
        if op == "norm_grad":
            return {"op": op, "tokens": tokens, "dim": dim, "src": src, "grad": rng.choice(["f32", half, half])}
        dst = rng.choice([half, half, "e4m3", "f32"])
        return {"op": op, "tokens": tokens, "dim": dim, "src": src, "res": rng.choice([half, half, "f32", "none"]), "dst": dst,
                "group": rng.choice([0, 32, 64, 128, 256]) if dst == "e4m3" else 0}
    vocab = rng.choice([_log(rng, 1000, 262144), 128 * _log(rng, 8, 2048), 64 * _log(rng, 16, 4096)])
    if op == "logits":
        rows = _log(rng, 1, min(2048, (1 << 27) // vocab))
        dst = rng.choice(["none", "f32", half])
        if dst == half and src == "f32":
            dst = "f32"
        return {"op": op, "rows": rows, "vocab": vocab, "src": src, "dst": dst, "history": rng.choice([0, _log(rng, 1, 16384)]),
                "biases": rng.choice([0, 0, _log(rng, 1, 300)]), "mask": rng.choice(["none", "some", "all"]),
                "pick": dst == "none" or rng.random() < 0.5}
    rows = _log(rng, 1, min(8192, (1 << 28) // vocab))
    return {"op": op, "rows": rows, "vocab": vocab, "src": src, "grad": "none" if op == "distill_eval" else rng.choice(["f32", half, half]) if src == "f32" else half,
            "top": _log(rng, 1, min(256, vocab)), "temperature": rng.choice([1.0, 1.0, 2.0, 0.7]), "normalize": rng.random() < 0.6}


def work(case):
    if case["op"] == "norm":
        n = case["tokens"] * case["dim"]
        res = 0 if case["res"] == "none" else 2 * SIZE[case["res"]]
        scales = case["tokens"] * _groups(case) * 4 if case["dst"] == "e4m3" else 0
        return {"bytes": n * (SIZE[case["src"]] + res + SIZE[case["dst"]]) + scales + 4 * case["dim"], "flops": 6 * n}
    if case["op"] == "norm_grad":
        n = case["tokens"] * case["dim"]
        return {"bytes": n * (SIZE[case["src"]] + 3 * SIZE[case["grad"]]) + 8 * case["dim"], "flops": 12 * n}
    n = case["rows"] * case["vocab"]
    if case["op"] == "logits":
        out = 0 if case["dst"] == "none" else SIZE[case["dst"]]
        masks = {"none": 0, "some": -(-case["rows"] // 3), "all": case["rows"]}[case["mask"]]
        return {"bytes": n * (SIZE[case["src"]] + out) + masks * 4 * -(-case["vocab"] // 32) + case["rows"] * (4 * case["history"] + 8 * case["biases"] + 36),
                "flops": 3 * n}
    out = 0 if case["grad"] == "none" else SIZE[case["grad"]]
    return {"bytes": n * (SIZE[case["src"]] + out) + case["rows"] * (case["top"] * 8 + 12), "flops": n * (4 if out == 0 else 8)}


def _groups(case):
    return -(-case["dim"] // case["group"]) if case["group"] else 1


# ---------------------------------------------------------------------------------------------- inputs
def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": dict(case)}
    {"norm": _prepare_norm, "norm_grad": _prepare_norm, "logits": _prepare_logits}.get(case["op"], _prepare_distill)(case, g, s)
    return s


def _prepare_norm(case, g, s):
    t, dim = case["tokens"], case["dim"]
    x = _randn(g, t, dim)
    x *= torch.exp(0.5 * _randn(g, dim))                                 # channels of uneven size
    s["x"] = x.to(TYPES[case["src"]])
    s["weight"] = 1.0 + 0.2 * _randn(g, dim)
    if case["op"] == "norm_grad":
        grad = TYPES[case["grad"]]
        s["dy"], s["dh"] = _randn(g, t, dim).to(grad), _randn(g, t, dim).to(grad)
        s["dx"] = torch.zeros(t, dim, dtype=grad, device="cuda")
        s["dweight"] = torch.zeros(dim, device="cuda")
        return
    s["residual"], s["h"] = None, None
    if case["res"] != "none":
        s["residual"] = (2.0 * _randn(g, t, dim)).to(TYPES[case["res"]])
        s["h"] = torch.zeros_like(s["residual"])
    s["y"] = torch.zeros(t, dim, dtype=TYPES[case["dst"]], device="cuda")
    s["scale"] = torch.zeros(t, _groups(case), device="cuda") if case["dst"] == "e4m3" else None


def _spread(g, rows, n, vocab):
    """n different tokens of each row."""
    step = torch.randint(1, max(2, vocab // max(n, 1)), (rows, 1), generator=g, device="cuda")
    first = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
    return ((first + step * torch.arange(n, device="cuda")) % vocab).to(torch.int32)


def _prepare_logits(case, g, s):
    rows, vocab, n = case["rows"], case["vocab"], case["history"]
    s["logits"] = (2.5 * _randn(g, rows, vocab) - 1.0).to(TYPES[case["src"]])
    s["out"] = None if case["dst"] == "none" else torch.zeros(rows, vocab, dtype=TYPES[case["dst"]], device="cuda")
    s["token"] = torch.zeros(rows, dtype=torch.int32, device="cuda") if case["pick"] else None
    s["lse"] = torch.zeros(rows, device="cuda") if case["pick"] else None
    s["history"], s["repetition"], s["frequency"], s["presence"] = None, None, None, None
    if n:
        # tokens come again like words do; -1 behind the last of a request
        s["history"] = (vocab * _rand(g, rows, n) ** 4).long().clamp(max=vocab - 1).to(torch.int32)
        s["history_len"] = torch.randint(n // 2, n + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
        s["history"].masked_fill_(torch.arange(n, device="cuda") >= s["history_len"][:, None], -1)
        s["prompt_len"] = (s["history_len"] * _rand(g, rows)).to(torch.int32)
        s["repetition"] = 1.0 + 0.5 * _rand(g, rows)
        s["frequency"], s["presence"] = 0.4 * _rand(g, rows), 0.6 * _rand(g, rows)
    s["bias"] = None
    if case["biases"]:
        many = min(case["biases"], vocab)
        s["bias"] = (torch.arange(rows + 1, device="cuda", dtype=torch.int32) * many, _spread(g, rows, many, vocab).flatten(),
                     4.0 * _randn(g, rows * many))
    s["mask"], s["mask_row"] = None, None
    if case["mask"] != "none":
        # half of the grammars' states allow a handful of tokens, half of them most
        s["mask_row"] = torch.arange(rows, device="cuda", dtype=torch.int32)
        masks = rows
        if case["mask"] == "some":
            masks = -(-rows // 3)
            s["mask_row"] = torch.where(s["mask_row"] % 3 == 0, s["mask_row"] // 3, torch.full_like(s["mask_row"], -1))
        words = -(-vocab // 32)
        share = torch.where(_rand(g, masks, 1) < 0.5, 20.0 / vocab, 0.9)
        s["mask"] = torch.zeros(masks, words, dtype=torch.int32, device="cuda")
        for bit in range(32):
            s["mask"] |= (_rand(g, masks, words) < share).to(torch.int32) << bit
        s["mask"][:, 0] |= 2


def _prepare_distill(case, g, s):
    rows, vocab, k = case["rows"], case["vocab"], case["top"]
    x = 2.0 * _randn(g, rows, vocab)
    t = torch.sort(3.0 * _randn(g, rows, k), dim=1, descending=True).values + 9.0
    s["teacher_token"] = _spread(g, rows, k, vocab)
    x.scatter_(1, s["teacher_token"].long(), t + 1.5 * _randn(g, rows, k))    # a student that has learnt something
    s["logits"] = x.to(TYPES[case["src"]])
    # as given they are logarithms of probabilities, which leave some of the mass to the tokens that are not listed
    s["teacher_logit"] = t if case["normalize"] else t - torch.logsumexp(t, 1, keepdim=True) - 0.1 * _rand(g, rows, 1)
    # padding has no weight
    s["row_weight"] = torch.where(_rand(g, rows) < 0.2, 0.0, 1.0 / rows) if case["op"] == "distill_grad" else torch.full((rows,), 1.0 / rows, device="cuda")
    if case["grad"] == "f16":
        s["row_weight"] *= 1024.0                                        # the loss scale of a training program in FP16
    s["loss"] = torch.zeros(rows, device="cuda")
    s["lse"] = torch.zeros(rows, device="cuda")
    s["dlogits"] = None if case["grad"] == "none" else torch.zeros(rows, vocab, dtype=TYPES[case["grad"]], device="cuda")


# ---------------------------------------------------------------------------------------------- plain forms (32 bits)
def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    got = {}
    if s["residual"] is not None:
        h = h + s["residual"].float()
        got["h"] = h.to(TYPES[case["res"]])
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"]
    if case["dst"] != "e4m3":
        got["y"] = y.to(TYPES[case["dst"]])
        return got
    t, dim = y.shape
    n, width = _groups(case), case["group"] or dim
    z = torch.zeros(t, n * width, device="cuda")
    z[:, :dim] = y
    z = z.view(t, n, width)
    top = z.abs().amax(-1)
    got["scale"] = torch.where(top > 0, (top / TOP).clamp(min=LEAST_SCALE), torch.ones_like(top))
    got["y"] = (z / got["scale"][..., None]).clamp(-TOP, TOP).view(t, -1)[:, :dim].to(torch.float8_e4m3fn)
    return got


def _plain_norm_grad(s):
    h, dy = s["x"].float(), s["dy"].float()
    r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    n = h * r
    g = dy * s["weight"]
    dx = r * (g - n * (g * n).mean(-1, keepdim=True)) + s["dh"].float()
    return {"dx": dx.to(TYPES[s["case"]["grad"]]), "dweight": (dy * n).sum(0)}


def _plain_logits(s):
    case = s["case"]
    rows, vocab, n = case["rows"], case["vocab"], case["history"]
    z = s["logits"].float()
    if n:
        at = torch.arange(n, device="cuda")
        said = at < s["history_len"][:, None]
        token = torch.where(said, s["history"], torch.zeros_like(s["history"])).long()
        seen = torch.zeros(rows, vocab, dtype=torch.int32, device="cuda").scatter_add_(1, token, said.to(torch.int32))
        made = torch.zeros(rows, vocab, dtype=torch.int32, device="cuda").scatter_add_(1, token, (said & (at >= s["prompt_len"][:, None])).to(torch.int32))
        z = torch.where(seen > 0, torch.where(z > 0, z / s["repetition"][:, None], z * s["repetition"][:, None]), z)
        z = z - (made.float() * s["frequency"][:, None] + torch.where(made > 0, s["presence"][:, None], torch.zeros_like(z)))
    if s["bias"] is not None:
        ptr, token, value = s["bias"]
        b = torch.zeros(rows, vocab, device="cuda")
        z = z + b.scatter_(1, token.view(rows, -1).long(), value.view(rows, -1))
    if s["mask"] is not None:
        bits = (s["mask"][s["mask_row"].clamp(min=0).long()][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        bad = (bits.view(rows, -1)[:, :vocab] == 0) & (s["mask_row"] >= 0)[:, None]
        z = z.masked_fill(bad, -math.inf)
    got = {}
    if s["out"] is not None:
        got["out"] = z.to(TYPES[case["dst"]])
    if case["pick"]:
        top, at = z.max(-1, keepdim=True)[0], torch.argmax(z, -1)
        got["token"] = torch.where(torch.isneginf(top[:, 0]), -1, at).to(torch.int32)
        got["lse"] = torch.log(torch.exp(z - torch.where(torch.isneginf(top), torch.zeros_like(top), top)).sum(-1)) + top[:, 0]
    return got


def _plain_distill(s):
    case = s["case"]
    x = s["logits"].float()
    if case["temperature"] != 1.0:
        x = x / case["temperature"]
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    token = s["teacher_token"].long()
    t = s["teacher_logit"].float()
    if case["normalize"]:
        t = t / case["temperature"]
        most = t.amax(-1, keepdim=True)
        t = t - most - torch.log(torch.exp(t - most).sum(-1, keepdim=True))
    p = torch.exp(t)
    live = s["row_weight"] != 0
    loss = (p * (t - (x.gather(1, token) - lse))).sum(-1)
    got = {"loss": torch.where(live, loss, torch.zeros_like(loss))}
    if case["grad"] == "none":
        return got
    w = (s["row_weight"] / case["temperature"])[:, None]
    e *= w * p.sum(-1, keepdim=True) / total
    e.scatter_add_(1, token, -w * p)
    got["dlogits"] = e.to(TYPES[case["grad"]])
    return got


# ---------------------------------------------------------------------------------------------- the library's operators
def _own_norm(s):
    from paper_2609_19758_b200 import norm as N
    case = s["case"]
    N.add_rms_norm(s["x"], s["residual"], s["weight"], s["y"], residual_out=s["h"], scale=s["scale"], group=case["group"], eps=EPS)
    return {n: s[n] for n in ("h", "y", "scale") if s[n] is not None}


def _own_norm_grad(s):
    from paper_2609_19758_b200 import norm as N
    if "ws" not in s:                                        # kept by a training program from step to step
        s["ws"] = N.add_rms_norm_workspace(s["case"]["dim"])
    N.add_rms_norm_backward(s["x"], s["dy"], s["weight"], s["dx"], s["dweight"], s["ws"], dh=s["dh"], eps=EPS)
    return {"dx": s["dx"], "dweight": s["dweight"]}


def _own_logits(s):
    from paper_2609_19758_b200 import logits as L
    lists = {n: s[n] for n in ("history", "history_len", "prompt_len", "repetition", "frequency", "presence")} if s["history"] is not None else {}
    L.adjust_logits(s["logits"], s["out"], bias=s["bias"], mask=s["mask"], mask_row=s["mask_row"], token=s["token"], lse=s["lse"], **lists)
    return {n: s[n] for n in ("out", "token", "lse") if s[n] is not None}


def _own_distill(s):
    from paper_2609_19758_b200 import logits as L
    case = s["case"]
    how = {"temperature": case["temperature"], "normalize": case["normalize"]}
    if case["op"] == "distill_eval":
        L.distill_loss(s["logits"], s["teacher_token"], s["teacher_logit"], s["loss"], **how)
        return {"loss": s["loss"]}
    if case["op"] == "distill":
        L.distill_loss(s["logits"], s["teacher_token"], s["teacher_logit"], s["loss"], row_weight=s["row_weight"], dlogits=s["dlogits"], **how)
    else:
        L.distill_loss(s["logits"], s["teacher_token"], s["teacher_logit"], s["loss"], row_weight=s["row_weight"], lse=s["lse"], **how)
        L.distill_loss_backward(s["logits"], s["teacher_token"], s["teacher_logit"], s["lse"], s["row_weight"], s["dlogits"], **how)
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def run(state):
    op = state["case"]["op"]
    if op == "norm":
        return _own_norm(state) if own else _plain_norm(state)
    if op == "norm_grad":
        return _own_norm_grad(state) if own else _plain_norm_grad(state)
    if op == "logits":
        return _own_logits(state) if own else _plain_logits(state)
    return _own_distill(state) if own else _plain_distill(state)


# ---------------------------------------------------------------------------------------------- 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "logits": _exact_logits}.get(case["op"], _exact_distill)(case, s)


def _exact_norm(case, s):
    x = s["x"].double()
    got = {}
    if s["residual"] is not None:
        x += s["residual"].double()
        got["h"] = x
    power = torch.linalg.vector_norm(x, dim=1) ** 2 / case["dim"] + EPS
    y = x * (s["weight"].double()[None] / torch.sqrt(power)[:, None])
    if case["dst"] == "e4m3":
        width = case["group"] or case["dim"]
        parts = y.split(width, dim=1)
        got["scale"] = torch.stack([torch.linalg.vector_norm(part, math.inf, dim=1) / TOP for part in parts], 1)
        y = torch.cat([part / got["scale"][:, i, None] for i, part in enumerate(parts)], 1)
    got["y"] = y
    return got


def _exact_norm_grad(case, s):
    x, dy, w = s["x"].double(), s["dy"].double(), s["weight"].double()
    power = torch.einsum("td,td->t", x, x) / case["dim"] + EPS
    along = torch.einsum("td,d,td->t", dy, w, x) / case["dim"]
    dx = s["dh"].double() + dy * w / power.sqrt()[:, None] - x * (along / power ** 1.5)[:, None]
    return {"dx": dx, "dweight": torch.einsum("td,td,t->d", dy, x, power ** -0.5)}


def _exact_logits(case, s):
    z = s["logits"].double()
    if s["history"] is not None:
        for r in range(case["rows"]):
            said = s["history"][r, :int(s["history_len"][r])].long()
            seen = torch.unique(said)
            made, times = torch.unique(said[int(s["prompt_len"][r]):], return_counts=True)
            rep = s["repetition"][r].double()
            z[r, seen] = torch.minimum(z[r, seen] * rep, z[r, seen] / rep)   # rep >= 1 in these inputs: either way down
            z[r, made] -= s["frequency"][r].double() * times + s["presence"][r].double()
    if s["bias"] is not None:
        ptr, token, value = s["bias"]
        row = torch.bucketize(torch.arange(len(token), device="cuda", dtype=torch.int32), ptr[1:], right=True)
        z.index_put_((row, token.long()), value.double(), accumulate=True)
    if s["mask"] is not None:
        v = torch.arange(case["vocab"], device="cuda")
        for r, m in enumerate(s["mask_row"].tolist()):
            if m >= 0:
                z[r, (s["mask"][m][v // 32] >> (v % 32)) % 2 == 0] = -math.inf
    got = {}
    if s["out"] is not None:
        got["out"] = z
    if case["pick"]:
        got["token"], got["lse"] = None, torch.logsumexp(z, -1)
    return got


def _exact_distill(case, s):
    tau, n = case["temperature"], case["rows"]
    loss, dlogits = torch.zeros(n, dtype=torch.float64, device="cuda"), None
    if case["grad"] != "none":
        dlogits = torch.zeros(n, case["vocab"], dtype=torch.float64, device="cuda")
    for a in range(0, n, 512):
        b = min(n, a + 512)
        logq = torch.log_softmax(s["logits"][a:b].double() / tau, -1)
        t, token = s["teacher_logit"][a:b].double(), s["teacher_token"][a:b].long()
        logp = torch.log_softmax(t / tau, -1) if case["normalize"] else t
        w = s["row_weight"][a:b].double()
        loss[a:b] = torch.where(w != 0, (logp.exp() * (logp - logq.gather(1, token))).sum(1), 0.0)
        if dlogits is not None:
            p = torch.zeros_like(logq).scatter_(1, token, logp.exp())
            dlogits[a:b] = (w / tau)[:, None] * (p.sum(1, keepdim=True) * logq.exp() - p)
    return {"loss": loss} if dlogits is None else {"loss": loss, "dlogits": dlogits}
