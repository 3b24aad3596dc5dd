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
        dlogits = B.moe_balance_loss_backward(logits, expert_idx, weight, dloss, dscale, ctx.renormalize)
        return dlogits, None, None, None


def balance_loss(logits, expert_idx, coef: float = 0.01, renormalize: bool = True):
    """logits [T, E] (fp16, bf16 or fp32, contiguous), expert_idx int32 [T, k] as moe_gate_topk gives it (E: a pruned row)
    -> (expert_scale [T, k], loss [], counts int32 [E], prob_mean [E]); expert_scale and loss carry gradients.
    expert_idx may be written again before the backward pass; logits may not (torch raises)."""
    return _BalanceLoss.apply(logits, expert_idx, coef, renormalize)
