"""The router's balance loss for training with torch: gate scales, load-balance loss and per-expert counts of given logits, differentiable with
respect to the logits (moe_balance_loss and its backward pass, include/moe_wq.h)."""
from __future__ import annotations

import torch

from . import binding as B


class _BalanceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, expert_idx, coef, renormalize):
        loss, counts, prob_mean, scale, weight = B.moe_balance_loss(logits, expert_idx, coef, renormalize)
        # (a copy of the index: a layer routes the next batch into the same buffer, through a pointer that torch's version counter does not see)
        ctx.save_for_backward(logits, expert_idx.clone(), weight)
        ctx.renormalize = renormalize
        ctx.mark_non_differentiable(counts, prob_mean)
        ctx.set_materialize_grads(False)
        return scale, loss, counts, prob_mean

    @staticmethod
    def backward(ctx, dscale, dloss, _counts, _prob_mean):
        logits, expert_idx, weight = ctx.saved_tensors
        if dscale is None and dloss is None:
            return None, None, None, None
        dscale = None if dscale is None else dscale.contiguous()
        gradient = _Gradient.apply if torch.is_grad_enabled() else B.moe_balance_loss_backward
        return gradient(logits, expert_idx, weight, dloss, dscale, ctx.renormalize), None, None, None


class _Gradient(torch.autograd.Function):
    """The gradient where a graph of it is asked for: a second derivative is refused, not left out.  (torch's once_differentiable refuses only where the
    gradients that come in have a graph of their own; that of logits alone it drops.)"""

    @staticmethod
    def forward(ctx, logits, expert_idx, weight, dloss, dscale, renormalize):
        return B.moe_balance_loss_backward(logits, expert_idx, weight, dloss, dscale, renormalize)

    @staticmethod
    def backward(ctx, _ddlogits):
        raise B.MoeError("balance_loss has no second derivative")


def balance_loss(logits, expert_idx, coef: float = 0.01, renormalize: bool = True):
    """logits [T, E] (fp16, bf16 or fp32, contiguous), expert_idx int32 [T, k] as moe_gate_topk gives it (E: a pruned row)
    -> (expert_scale [T, k], loss [], counts int32 [E], prob_mean [E]); expert_scale and loss carry gradients.
    expert_idx may be written again before the backward pass; logits may not (torch raises)."""
    return _BalanceLoss.apply(logits, expert_idx, coef, renormalize)
