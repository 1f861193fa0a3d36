"""The end loss as autograd sees it: :func:`token_logprobs` and :func:`end_loss` over the library's kernels.

The saliencies are squares of the end loss' gradients (Section 3.1), so the calibration's backward pass starts here; the same log
probabilities, entropies and alternatives measure a quantised model.  No arithmetic happens in this module beyond adding up the
tokens' losses."""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import api


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, top):
        logp, entropy, stats, top_logp, top_ids = api.gq_token_logprobs(logits, targets, top=top)
        ctx.save_for_backward(logits, targets, stats, entropy)
        ctx.set_materialize_grads(False)
        outside = [t for t in (top_logp, top_ids) if t is not None]
        ctx.mark_non_differentiable(*outside)
        return logp, entropy, top_logp, top_ids

    @staticmethod
    @once_differentiable
    def backward(ctx, d_logp, d_entropy, _d_top_logp, _d_top_ids):
        logits, targets, stats, entropy = ctx.saved_tensors
        if d_logp is None and d_entropy is None:
            return None, None, None
        d_logp, d_entropy = (None if d is None else d.float().contiguous() for d in (d_logp, d_entropy))
        return api.gq_token_logprobs_grad(logits, targets, stats, entropy, d_logp, d_entropy), None, None


def token_logprobs(logits: torch.Tensor, targets: torch.Tensor, top: int = 0):
    """``(logp, entropy, top_logp, top_ids)`` of ``logits`` ``[..., vocab]`` and ``targets`` ``[...]``, all of the targets' shape (the last two
    with a trailing ``top``, or ``None``).  A target outside ``[0, vocab)`` does not count: log probability 0, no gradient.
    ``logp`` and ``entropy`` carry gradients to the logits, the alternatives do not."""
    vocab = logits.shape[-1]
    if logits.shape[:-1] != targets.shape:
        raise ValueError("targets must have the shape of logits without its last dimension")
    rows = logits.reshape(-1, vocab)
    if (vocab > 1 and rows.stride(1) != 1) or (rows.shape[0] > 1 and rows.stride(0) < vocab):      # (rows that share memory: expanded ones)
        rows = rows.contiguous()
    logp, entropy, top_logp, top_ids = _TokenLogprobs.apply(rows, targets.reshape(-1).contiguous(), int(top))
    shape = targets.shape
    if top:
        top_logp, top_ids = top_logp.view(*shape, top), top_ids.view(*shape, top)
    return logp.view(shape), entropy.view(shape), top_logp, top_ids


def end_loss(logits: torch.Tensor, targets: torch.Tensor, weight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Minus the sum of the targets' log probabilities (fp32 scalar), tokens weighted by ``weight`` if given.  The sum, not the mean: a
    token's gradient then does not depend on the batch that it is in."""
    logp = token_logprobs(logits, targets)[0]
    return -(logp.sum() if weight is None else (logp * weight).sum())
