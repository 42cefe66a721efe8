"""A decoder whose projections are verified: ``python -m paper_2609_19758_b200.decoder``.

Attention layers (``attention_layer.py``) joined by ``norm.add_rms_norm``, which takes the FP32 accumulator of a layer's output
projection to the residual stream and makes the next layer's input in the same pass, and a head whose accumulator goes, un-narrowed
and probed, through ``logits.adjust_logits`` to the next tokens, or through ``logits.distill_loss`` to the gradients of a training
step.  Verdicts are accumulated on the device and read once per step; a dirty step is retracted and repeated.
"""
from __future__ import annotations

import argparse
from typing import List, Optional, Sequence

import torch

from . import fpsk, harness, logits, norm
from .attention_layer import VerifiedAttention


MOST_PROBED = 1 << 17      # columns of a product that are probed together, and half of the channels that it sums over (a probe takes 1.15 times as many)


def _parts(n: int, most: int):
    """The ranges of 0 .. n of at most `most`, as long as each other but for multiples of 8."""
    step = -(-n // (-(-n // most)))
    step += -step % 8
    return [(i, min(n, i + step)) for i in range(0, n, step)]


class VerifiedHead:
    """The product of a model's last states with a weight (hidden, vocab), verified, and what follows it."""

    def __init__(self, weight: torch.Tensor):
        self.weight = weight
        with torch.cuda.device(weight.device):
            self.state = fpsk.new_probe_state(weight.device)
        self.result = fpsk.new_probe_result(weight.device)
        self.status = torch.zeros(1, dtype=torch.int32, device=weight.device)
        self.probe_ws = []                                             # (the last one serves; graphs may hold those that it has replaced)

    def _workspace(self, k: int, n: int) -> torch.Tensor:
        """One for all products: training steps of many lengths have as many shapes of the weight's gradient.  Each is twice the one before at
        least, so that all together are less than twice the last."""
        held = self.probe_ws[-1].numel() if self.probe_ws else 0
        if held < int(fpsk.lib().fpsk_probe_workspace_bytes(1, k, n)):  # (it does not depend on the rows of the other operand)
            self.probe_ws.append(fpsk.probe_workspace(1, k, n, device=self.weight.device, room=2 * held))
        return self.probe_ws[-1]

    def product(self, a: torch.Tensor, b: torch.Tensor, fault=None) -> torch.Tensor:
        """a b with the accumulator in FP32, probed; `fault`: (row, column, what to add), for trying the probe."""
        if b.shape[0] > 2 * MOST_PROBED:                               # (a sum over a wide vocabulary: parts of it, added up)
            (first, last), *rest = _parts(b.shape[0], 2 * MOST_PROBED)
            c = self.product(a[:, first:last], b[first:last], fault)
            for first, last in rest:
                c += self.product(a[:, first:last], b[first:last])
            return c
        c = harness.vendor_gemm_fp32(a, b)
        if fault is not None:
            c[fault[0], fault[1]] += fault[2]
        with torch.cuda.device(b.device):                              # (the probe runs on the current device)
            for first, last in _parts(b.shape[1], MOST_PROBED):
                fpsk.probe(a, b[:, first:last], c[:, first:last], self._workspace(b.shape[0], last - first), self.result)
                fpsk.probe_accumulate(self.result, self.state)
        return c

    def next_tokens(self, x: torch.Tensor, fault=None, **how) -> torch.Tensor:
        """The tokens (int32) of the largest logits of the states x (rows, hidden), after the penalties, biases and masks of
        ``logits.adjust_logits`` that `how` names."""
        token = torch.empty(x.shape[0], dtype=torch.int32, device=x.device)
        logits.adjust_logits(self.product(x, self.weight, fault), token=token, status=self.status, **how)
        return token

    def distill(self, x: torch.Tensor, teacher_token: torch.Tensor, teacher_logit: torch.Tensor, row_weight: Optional[torch.Tensor] = None,
                temperature: float = 1.0, normalize: bool = True):
        """A training step's share of the head: the losses of the states x against a teacher's top logits, and the FP32 gradients of
        sum(row_weight * loss) with respect to x and the weight.  Three products, all verified; the gradient of the logits is made
        in the operands' type in the pass that makes the losses."""
        c = self.product(x, self.weight)
        # FP16 ends at 6e-8, which probabilities times the weights of a mean are below: the logits' gradient is made for weights whose
        # largest, by the temperature, is 2^8 to 2^9, and the products are scaled back.  (Powers of two, made on the device.)
        back = None
        if x.dtype == torch.float16:
            most = torch.ones(1, device=x.device) if row_weight is None else row_weight.abs().amax().view(1)
            scale = torch.exp2(8 - torch.floor(torch.log2((most / temperature).clamp(2.0 ** -100, 2.0 ** 100))))
            row_weight, back = scale.expand(x.shape[0]).contiguous() if row_weight is None else row_weight * scale, 1 / scale
        loss = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
        dlogits = torch.empty(c.shape, dtype=x.dtype, device=x.device)
        logits.distill_loss(c, teacher_token, teacher_logit, loss, row_weight=row_weight, dlogits=dlogits, temperature=temperature, normalize=normalize,
                            status=self.status)
        # The probe compares the columns' sums of an error with their mean: the products are laid out so that the logits' gradient, whose
        # columns differ by orders of magnitude between tokens that are listed and others, has the rows, not the columns.
        dx, dw = self.product(dlogits, self.weight.t().contiguous()), self.product(dlogits.t().contiguous(), x).t()
        if back is not None:
            dx, dw = dx.mul_(back), dw.mul_(back)
        return loss, dx, dw

    def fired(self) -> bool:
        """Whether any product since the last call was dirty.  What the kernels reported since then is raised."""
        s = fpsk.read_probe_state(self.state)
        with torch.cuda.device(self.state.device):
            fpsk.reset_probe_state(self.state)
        reported = int(self.status)
        if reported != fpsk.STATUS_OK:
            self.status.zero_()
            raise fpsk.FpskError(reported, "verified head")
        return bool(s.fired_any)


class VerifiedDecoder:
    """Token embeddings (vocab, hidden), attention layers with a norm weight (hidden,) in front of each, a last norm weight, a head."""

    def __init__(self, embedding: torch.Tensor, layers: Sequence[VerifiedAttention], norm_weights: Sequence[torch.Tensor], head: VerifiedHead, eps: float = 1e-6):
        if not layers or len(norm_weights) != len(layers) + 1:
            raise ValueError("a norm weight for each layer, of which there is one at least, and one for the head")
        self.embedding, self.layers, self.norm_weights, self.head, self.eps = embedding, list(layers), list(norm_weights), head, eps
        self.status = torch.zeros(1, dtype=torch.int32, device=embedding.device)
        self.stepped = 0

    def open(self) -> int:
        """A new sequence."""
        seqs = [layer.pages.open() for layer in self.layers]
        if len(set(seqs)) > 1:                                         # (one number stands for all layers: another's sequence would be written to)
            for layer, seq in zip(self.layers, seqs):
                layer.pages.close(seq)
            raise RuntimeError("the layers have had different numbers of sequences: they serve one decoder, and in one place")
        return seqs[0]

    def close(self, seq: int) -> None:
        for layer in self.layers:
            layer.pages.close(seq)

    def step(self, tokens: torch.Tensor, seqs: Sequence[int], new: Sequence[int], fault=None) -> torch.Tensor:
        """The new tokens (packed, `new` of each sequence) through the layers: the last states (tokens, hidden) for the head.  `fault`: an
        entry of the first layer's accumulator, see VerifiedAttention.  A step that is refused changes nothing; a token outside the
        vocabulary is raised with the verdicts."""
        if tokens.dim() != 1 or tokens.shape[0] != sum(new) or tokens.shape[0] == 0 or tokens.device != self.embedding.device:
            raise ValueError(f"tokens: ({sum(new)},) on {self.embedding.device} expected, at least one")
        most = self.embedding.shape[0] - 1
        bad = ((tokens < 0) | (tokens > most)).any()                   # (told with the verdicts: the host does not know the tokens)
        torch.maximum(self.status, bad.to(torch.int32) * fpsk.ERR_PARAM, out=self.status)
        h = self.embedding[tokens.long().clamp(0, most)]               # the residual stream
        x = torch.empty_like(h)
        norm.add_rms_norm(h, None, self.norm_weights[0], x, eps=self.eps, status=self.status)
        self.stepped = 0
        try:
            for layer, weight in zip(self.layers, self.norm_weights[1:]):
                c = layer.step(x, seqs, new, fault)
                self.stepped += 1
                fault = None
                norm.add_rms_norm(c, h, weight, x, residual_out=h, eps=self.eps, status=self.status)
        except BaseException:
            self.retract()
            raise
        return x

    def retract(self) -> None:
        """Takes the last step's tokens out of the layers' caches again."""
        for layer in self.layers[:self.stepped]:
            layer.retract()
        self.stepped = 0

    def fired(self) -> bool:
        """Whether any product since the last call was dirty (one host read a layer).  What the kernels reported is raised, after all verdicts
        have been read: the next call's are those of what comes next."""
        fired, raised = False, None
        for part in [*self.layers, self.head]:
            try:
                fired |= part.fired()
            except fpsk.FpskError as e:
                raised = raised or e
        reported = int(self.status)
        if reported != fpsk.STATUS_OK:
            self.status.zero_()
            raised = raised or fpsk.FpskError(reported, "verified decoder")
        if raised is not None:
            raise raised
        return fired

    def generate(self, prompts: Sequence[Sequence[int]], steps: int, repetition: float = 1.0, frequency: float = 0.0, presence: float = 0.0,
                 mask: Optional[torch.Tensor] = None, fault_at: int = -1) -> List[List[int]]:
        """Greedy tokens for the prompts, `steps` of each.  mask: one row of allowed tokens for all (int32 words, see
        ``logits.adjust_logits``).  A step that fired is retracted and repeated, a second time raises; `fault_at`: the step that meets a
        corrupted accumulator entry, for trying that."""
        dev, n = self.embedding.device, len(prompts)
        if n == 0 or any(len(p) == 0 for p in prompts):
            raise ValueError("prompts of at least one token each")
        if any(not 0 <= t < self.embedding.shape[0] for p in prompts for t in p):
            raise ValueError("a token outside the vocabulary")
        width = max(len(p) for p in prompts) + steps
        history = torch.full((n, width), -1, dtype=torch.int32)
        for i, p in enumerate(prompts):
            history[i, :len(p)] = torch.tensor(list(p), dtype=torch.int32)
        history = history.to(dev)
        prompt_len = torch.tensor([len(p) for p in prompts], dtype=torch.int32, device=dev)
        length = prompt_len.clone()
        rows = torch.arange(n, device=dev)
        how = dict(history=history, history_len=length, prompt_len=prompt_len, repetition=torch.full((n,), repetition, device=dev),
                   frequency=torch.full((n,), frequency, device=dev), presence=torch.full((n,), presence, device=dev))
        if mask is not None:
            how.update(mask=mask.view(1, -1), mask_row=torch.zeros(n, dtype=torch.int32, device=dev))
        seqs = [self.open() for _ in prompts]
        try:
            tokens, new = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device=dev), [len(p) for p in prompts]
            for k in range(steps):
                for attempt in range(2):
                    x = self.step(tokens, seqs, new, (0, 0, 30.0) if k == fault_at and attempt == 0 else None)
                    last = torch.cumsum(torch.tensor(new, device=dev), 0) - 1
                    picked = self.head.next_tokens(x[last], **how)
                    if not self.fired():
                        break
                    self.retract()
                else:
                    raise RuntimeError("a step fired twice")
                if bool((picked < 0).any()):
                    raise RuntimeError("the mask allows nothing")
                history[rows, length.long()] = picked
                length += 1
                tokens, new = picked, [1] * n
            return [row[p:p + steps] for row, p in zip(history.tolist(), prompt_len.tolist())]
        finally:
            for seq in seqs:
                self.close(seq)


def demo_decoder(vocab: int = 4096, hidden: int = 1024, layers: int = 2, hq: int = 8, hk: int = 2, dim: int = 128, dtype=torch.bfloat16, seed: int = 0) -> VerifiedDecoder:
    """A decoder with random weights."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g, device="cuda")).to(dtype)

    def weight():
        return 1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")

    attention = [VerifiedAttention(rand(hidden, (hq + 2 * hk) * dim, scale=hidden ** -0.5), rand(hq * dim, hidden, scale=(hq * dim) ** -0.5), hq, hk, dim,
                                   torch.ones(dim, device="cuda"), torch.ones(dim, device="cuda")) for _ in range(layers)]
    return VerifiedDecoder(rand(vocab, hidden), attention, [weight() for _ in range(layers + 1)], VerifiedHead(rand(hidden, vocab, scale=hidden ** -0.5)))


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__)
    p.add_argument("--steps", type=int, default=8)
    p.add_argument("--prompts", default="5,1,12", help="lengths of the prompts")
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--repetition", type=float, default=1.2)
    a = p.parse_args()
    d = demo_decoder(layers=a.layers)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, d.embedding.shape[0], (int(n),), generator=g).tolist() for n in a.prompts.split(",")]
    plain = d.generate(prompts, a.steps, repetition=a.repetition)
    again = d.generate(prompts, a.steps, repetition=a.repetition, fault_at=a.steps // 2)
    for q, t in zip(prompts, plain):
        print(f"prompt of {len(q)}: {t}")
    print(f"with a corrupted accumulator entry in step {a.steps // 2}, retracted and repeated: {'the same tokens' if again == plain else 'OTHER TOKENS'}")


if __name__ == "__main__":
    main()
