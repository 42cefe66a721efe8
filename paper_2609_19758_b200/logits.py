"""What is done to the logits of a verified head (``include/fpsk_decoder.h``): penalties, biases and grammar masks with the greedy token,
and the loss against a teacher's top logits with its gradient.

Argument marshalling only, like ``attention.py``: every step runs inside the CUDA library, asynchronously on the given (or the
current) stream of the tensors' device.  Outputs are the caller's tensors; wrong shapes, types, devices or strides raise ValueError
or TypeError, what the library refuses raises FpskError.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable

from . import attention as A


def adjust_logits(logits: torch.Tensor, out: Optional[torch.Tensor] = None, history: Optional[torch.Tensor] = None,
                  history_len: Optional[torch.Tensor] = None, prompt_len: Optional[torch.Tensor] = None,
                  repetition: Optional[torch.Tensor] = None, frequency: Optional[torch.Tensor] = None,
                  presence: Optional[torch.Tensor] = None, bias: Optional[Tuple[torch.Tensor, torch.Tensor, torch.Tensor]] = None,
                  mask: Optional[torch.Tensor] = None, mask_row: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None, stream=None) -> None:
    """logits (rows, vocab) adjusted in FP32: tokens of the row's history (int32 (rows, width), the first history_len of them, the first
    prompt_len of those the prompt's; -1 is passed over) have z > 0 divided, else multiplied by repetition, and are lowered by
    frequency * c + presence where they come c > 0 times behind the prompt; bias = (first entries of the rows (rows + 1,), tokens, values)
    is added; tokens whose bit of the row's mask (int32 (masks, ceil(vocab / 32)), row r has mask_row[r], -1: none) is 0 become -inf.
    The result goes to out (which may be logits), rounded once; token (int32) gets the largest one's token, -1 where nothing is allowed, lse the
    log-sum-exp."""
    b = A._binding or A._bind()
    first, tokens, values = bias if bias is not None else (None, None, None)
    A._check(b.adjust_logits(logits, out, history, history_len, prompt_len, repetition, frequency, presence, first, tokens, values, mask,
                             mask_row, token, lse, status, A._stream(b.device(logits), stream)), "fpsk_adjust_logits")


def distill_loss(logits: torch.Tensor, teacher_token: torch.Tensor, teacher_logit: torch.Tensor, loss: torch.Tensor,
                 row_weight: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, normalize: bool = True, status: Optional[torch.Tensor] = None, stream=None,
                 sums: Optional[torch.Tensor] = None) -> None:
    """loss (rows,): sum_j p_j (log p_j - log q_j) of each row of logits (rows, vocab), q = softmax(logits / temperature), against the
    teacher's logits for the tokens teacher_token (rows, top): p = softmax(teacher_logit / temperature) over them, or exp(teacher_logit)
    with normalize=False (logarithms of probabilities).  Tokens outside the vocabulary (-1) are left out.  dlogits (rows, vocab) gets the gradient of
    sum(row_weight * loss) in the same launch; it may be logits.  Rows of weight 0 are not read: loss 0, gradient 0.  lse (rows,) and sums
    (rows, 2), both FP32, keep the rows' log-sum-exps for distill_loss_backward."""
    b = A._binding or A._bind()
    A._check(b.distill_loss(logits, teacher_token, teacher_logit, loss, row_weight, lse, dlogits, temperature, normalize, sums, status,
                            A._stream(b.device(logits), stream)), "fpsk_distill_loss")


def distill_loss_backward(logits: torch.Tensor, teacher_token: torch.Tensor, teacher_logit: torch.Tensor, lse: Optional[torch.Tensor],
                          dloss: torch.Tensor, dlogits: torch.Tensor, temperature: float = 1.0, normalize: bool = True,
                          status: Optional[torch.Tensor] = None, stream=None, sums: Optional[torch.Tensor] = None) -> None:
    """The gradient of distill_loss alone, from the sums (or the lse, which costs its rounding) of the forward pass and the gradients dloss
    (rows,) of the rows' losses."""
    b = A._binding or A._bind()
    A._check(b.distill_loss_backward(logits, teacher_token, teacher_logit, None, dloss, lse, dlogits, temperature, normalize, sums, status,
                                     A._stream(b.device(logits), stream)), "fpsk_distill_loss_backward")


class DistillLoss(torch.autograd.Function):
    """distill_loss for autograd: ``apply(logits, teacher_token, teacher_logit, temperature, normalize, row_weight=None)`` returns the rows'
    losses.  Rows whose row_weight is 0 (padding) are not read: their loss and gradient are 0, whatever they hold; the other losses come
    as they are, for the caller to weight.  The teacher gets no gradient; a second derivative is refused."""

    @staticmethod
    def forward(ctx, logits, teacher_token, teacher_logit, temperature, normalize, row_weight=None):
        loss, sums = (torch.empty(logits.shape[0], *more, dtype=torch.float32, device=logits.device) for more in ((), (2,)))
        distill_loss(logits, teacher_token, teacher_logit, loss, row_weight=row_weight, temperature=temperature, normalize=normalize, sums=sums)
        ctx.save_for_backward(logits, teacher_token, teacher_logit, sums, row_weight)
        ctx.more = (temperature, normalize)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        logits, teacher_token, teacher_logit, sums, row_weight = ctx.saved_tensors
        dloss = dloss.float().contiguous()
        if row_weight is not None:
            dloss = dloss.masked_fill(row_weight == 0, 0.0)
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        distill_loss_backward(logits, teacher_token, teacher_logit, None, dloss, dlogits, *ctx.more, sums=sums)
        return dlogits, None, None, None, None, None
