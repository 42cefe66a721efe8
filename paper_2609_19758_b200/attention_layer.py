"""An attention layer whose projections are verified: ``python -m paper_2609_19758_b200.attention_layer``.

The QKV projection is a vendor GEMM with its FP32 accumulator delivered.  The probe checks it; then the accumulator itself is
read by ``paged_append`` (queries and keys normed and rotated, keys and values written to the pages of the cache, rounded
once), ``paged_attention`` runs the new tokens over the cache, and the output projection is checked like the first.  Verdicts
are accumulated on the device and read once per step; a dirty step is retracted and repeated.
"""
from __future__ import annotations

import argparse
from typing import List, Optional, Sequence

import torch

from . import attention as A
from . import fpsk, harness


class PageTable:
    """Hands out the pages of a cache and keeps the table of every sequence (host side)."""

    def __init__(self, n_pages: int, page_size: int):
        self.free = list(range(n_pages))[::-1]
        self.page_size = page_size
        self.rows: List[List[int]] = []
        self.length: List[int] = []

    def open(self) -> int:
        self.rows.append([])
        self.length.append(0)
        return len(self.rows) - 1

    def extend(self, seq: int, tokens: int) -> None:
        self.extend_all([seq], [tokens])

    def extend_all(self, seqs: Sequence[int], tokens: Sequence[int], most: Optional[int] = None) -> None:
        """Room for the new tokens of several sequences, of at most `most` tokens each: for all of them, or an exception and none."""
        if len(seqs) != len(tokens) or len(set(seqs)) != len(seqs):
            raise ValueError("a number of tokens for each sequence, each sequence once")
        if any(not 0 <= b < len(self.rows) for b in seqs) or any(n < 0 for n in tokens):
            raise ValueError("an unknown sequence, or a negative number of tokens")
        if most is not None and any(self.length[b] + n > most for b, n in zip(seqs, tokens)):
            raise ValueError(f"a sequence of more than {most} tokens")
        wanted = [-(-(self.length[b] + n) // self.page_size) - len(self.rows[b]) for b, n in zip(seqs, tokens)]
        if sum(wanted) > len(self.free):
            raise RuntimeError("the cache is full")
        for b, n, pages in zip(seqs, tokens, wanted):
            self.rows[b] += [self.free.pop() for _ in range(pages)]
            self.length[b] += n

    def retract(self, seqs: Sequence[int], tokens: Sequence[int]) -> None:
        """Takes the last tokens of the sequences out again, and their pages where nothing is left on them."""
        if len(seqs) != len(tokens) or len(set(seqs)) != len(seqs):
            raise ValueError("a number of tokens for each sequence, each sequence once")
        if any(not 0 <= b < len(self.rows) for b in seqs) or any(not 0 <= n <= self.length[b] for b, n in zip(seqs, tokens)):
            raise ValueError("an unknown sequence, or more tokens than it has")
        for b, n in list(zip(seqs, tokens))[::-1]:                     # (the reverse of extend_all, page for page)
            self.length[b] -= n
            while (len(self.rows[b]) - 1) * self.page_size >= self.length[b] and self.rows[b]:
                self.free.append(self.rows[b].pop())

    def close(self, seq: int) -> None:
        self.free += self.rows[seq][::-1]
        self.rows[seq], self.length[seq] = [], 0


class VerifiedAttention:
    """One attention layer over a paged cache.  qkv_weight (hidden, (hq + 2 hk) dim) and out_weight (hq dim, hidden) are the
    B operands of the two products."""

    def __init__(self, qkv_weight: torch.Tensor, out_weight: torch.Tensor, hq: int, hk: int, dim: int, q_weight=None, k_weight=None,
                 n_pages: int = 256, page_size: int = 16, n_pos: int = 8192, rot_dim: Optional[int] = None, eps: float = 1e-6):
        self.qkv_weight, self.out_weight = qkv_weight, out_weight
        self.hq, self.hk, self.dim, self.eps = hq, hk, dim, eps
        self.q_weight, self.k_weight = q_weight, k_weight
        dev, dt = qkv_weight.device, qkv_weight.dtype
        self.cache = A.PagedCache(*(torch.zeros(n_pages, page_size, hk, dim, dtype=dt, device=dev) for _ in range(2)))
        self.pages = PageTable(n_pages, page_size)
        self.cos, self.sin = A.rotary_tables(n_pos, dim if rot_dim is None else rot_dim, device=dev)
        self.ws = A.attention_workspace(dev)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.state = fpsk.new_probe_state(dev)
        self.result = fpsk.new_probe_result()
        self.probe_ws = {}
        self.last = None                                               # sequences and new tokens of the last step

    def _verified(self, x: torch.Tensor, w: torch.Tensor, fault=None) -> torch.Tensor:
        """x w with the accumulator in FP32, probed; `fault`: (row, column, what to add), for trying the probe."""
        c = harness.vendor_gemm_fp32(x, w)
        if fault is not None:
            c[fault[0], fault[1]] += fault[2]
        key = (w.shape[0], w.shape[1])
        if key not in self.probe_ws:                                   # (its size does not depend on the rows of x)
            self.probe_ws[key] = fpsk.probe_workspace(1, *key)
        fpsk.probe(x, w, c, self.probe_ws[key], self.result)
        fpsk.probe_accumulate(self.result, self.state)
        return c

    def step(self, x: torch.Tensor, seqs: Sequence[int], new: Sequence[int], fault=None) -> torch.Tensor:
        """x (tokens, hidden): the new tokens of the sequences `seqs`, `new` of each.  Returns the layer's output, FP32.  A step that is
        refused (ValueError, or RuntimeError when the cache is full) changes nothing."""
        w = self.qkv_weight
        if x.dim() != 2 or x.shape[1] != w.shape[0] or x.shape[0] != sum(new) or x.shape[0] == 0 or x.dtype != w.dtype or x.device != w.device:
            raise ValueError(f"x: ({sum(new)}, {w.shape[0]}) {w.dtype} on {w.device} expected, at least one token")
        self.pages.extend_all(seqs, new, most=self.cos.shape[0] if self.cos.shape[1] else None)
        try:
            out = self._step(x, seqs, new, fault)
        except BaseException:
            self.pages.retract(seqs, new)
            raise
        self.last = (list(seqs), list(new))
        return out

    def _step(self, x, seqs, new, fault):
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        kv = [self.pages.length[b] for b in seqs]
        width = max(max(len(self.pages.rows[b]) for b in seqs), 1)
        table = [self.pages.rows[b] + [-1] * (width - len(self.pages.rows[b])) for b in seqs]
        cu_q, kv_len, block_table = (torch.tensor(t, dtype=torch.int32).to(x.device) for t in (cu, kv, table))
        hq, hk, dim, n = self.hq, self.hk, self.dim, x.shape[0]
        c = self._verified(x, self.qkv_weight, fault)
        q, k, v = (t.unflatten(1, (-1, dim)) for t in c.split((hq * dim, hk * dim, hk * dim), dim=1))
        q_out = torch.empty(n, hq, dim, dtype=x.dtype, device=x.device)
        A.paged_append(self.cache, k, v, cu_q, kv_len, block_table, self.cos, self.sin, self.k_weight, q=q, q_out=q_out,
                       q_weight=self.q_weight, eps=self.eps, status=self.status)
        out = torch.empty_like(q_out)
        A.paged_attention(self.cache, q_out, out, cu_q, kv_len, block_table, self.ws, max(new), max(kv), status=self.status)
        return self._verified(out.flatten(1), self.out_weight)

    def retract(self) -> None:
        """Takes the last step's tokens out of the cache again, whose keys and values are there before the verdict is: a step that
        `fired` (or raised what the device reported) is retracted and repeated."""
        if self.last is None:
            raise RuntimeError("no step to retract")
        self.pages.retract(*self.last)
        self.last = None

    def fired(self) -> bool:
        """Whether any product since the last call was dirty (where a step is read on the host).  What the kernels of the append and the
        attention reported since then, a page outside the cache or a wait that gave up, is raised."""
        s = fpsk.read_probe_state(self.state)
        fpsk.reset_probe_state(self.state)
        reported = int(self.status)
        if reported != fpsk.STATUS_OK:
            self.status.zero_()
            self.ws = A.attention_workspace(self.ws.device)            # (a wait that gave up may leave its words)
            raise fpsk.FpskError(reported, "attention layer")
        return bool(s.fired_any)


def demo(hidden: int = 4096, hq: int = 32, hk: int = 8, dim: int = 128, prompts: Sequence[int] = (700, 123, 1), steps: int = 4,
         dtype=torch.bfloat16, seed: int = 0) -> dict:
    """Prompts, then decoding steps of all sequences at once, then a step with a corrupted accumulator entry."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    cols = (hq + 2 * hk) * dim
    layer = VerifiedAttention((rand(hidden, cols) * hidden ** -0.5).to(dtype), (rand(hq * dim, hidden) * (hq * dim) ** -0.5).to(dtype), hq, hk, dim,
                              1 + 0.1 * rand(dim), 1 + 0.1 * rand(dim))
    seqs = [layer.pages.open() for _ in prompts]
    inputs, outputs = [[] for _ in prompts], [[] for _ in prompts]

    def run(new, fault=None):
        x = rand(sum(new), hidden).to(dtype)
        y = layer.step(x, seqs, new, fault)
        for b, (xs, ys) in enumerate(zip(x.split(list(new)), y.split(list(new)))):
            inputs[b].append(xs)
            outputs[b].append(ys)
        return layer.fired()

    fired = [run(list(prompts))] + [run([1] * len(prompts)) for _ in range(steps)]
    faulty = run([1] * len(prompts), fault=(0, 5, 3.0))
    return {"layer": layer, "inputs": [torch.cat(t) for t in inputs], "outputs": [torch.cat(t) for t in outputs], "fired": fired, "fired_on_fault": faulty}


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__)
    p.add_argument("--steps", type=int, default=4)
    p.add_argument("--prompts", default="700,123,1")
    a = p.parse_args()
    r = demo(prompts=[int(t) for t in a.prompts.split(",")], steps=a.steps)
    print(f"prompts {a.prompts}, {a.steps} decoding steps: verdicts {[int(f) for f in r['fired']]}; with a corrupted accumulator entry: {int(r['fired_on_fault'])}")


if __name__ == "__main__":
    main()
