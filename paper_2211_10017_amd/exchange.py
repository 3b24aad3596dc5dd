"""Sorting tokens by expert and back as functions with gradients, for training with torch (moe_permute, moe_combine and their backward passes, include/moe_wq.h)."""
from __future__ import annotations

import torch

from . import binding as B


class Once(torch.autograd.Function):
    """A gradient where a graph of it is asked for: a second derivative is refused, not left out."""

    @staticmethod
    def forward(ctx, call, name, *tensors):
        ctx.name = name
        return call(*tensors)

    @staticmethod
    def backward(ctx, *_):
        raise B.MoeError("%s has no second derivative" % ctx.name)


def gradient(call, name, *tensors):
    """call(*tensors) in a backward pass."""
    return Once.apply(call, name, *tensors) if torch.is_grad_enabled() else call(*tensors)


def whole(t):
    """A gradient as the library reads it: contiguous, on 16 bytes.  (torch may hand over a part of a larger one, contiguous wherever it begins.)"""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


class _Permute(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, expert_idx, E):
        T, k = expert_idx.shape
        R, dev = T * k, x.device
        # (rows behind the last expert's are 0: what uses them as if they were rows must not meet what lay there)
        x_perm = torch.zeros((R, x.shape[1]), dtype=x.dtype, device=dev)
        perm_src, inv_perm = (torch.empty(R, dtype=torch.int32, device=dev) for _ in range(2))
        offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
        B.moe_permute(expert_idx, x, E, out=(x_perm, perm_src, inv_perm, offsets))
        ctx.save_for_backward(inv_perm.clone(), offsets[E:].clone())        # (copies: the index may be written again before the backward pass)
        ctx.sizes = T, k
        ctx.mark_non_differentiable(perm_src, inv_perm, offsets)
        return x_perm, perm_src, inv_perm, offsets

    @staticmethod
    def backward(ctx, dx_perm, *_):
        inv_perm, active = ctx.saved_tensors
        call = lambda g: B.moe_permute_backward(g, inv_perm, *ctx.sizes, active_rows=active)  # noqa: E731
        return gradient(call, "permute_tokens", whole(dx_perm)), None, None


def permute_tokens(x, expert_idx, E: int):
    """x [T, d], expert_idx int32 [T, k] (E: a pruned row) -> (x_perm [T * k, d], perm_src, inv_perm, expert_offsets); x_perm carries gradients, its rows behind the last expert's are 0."""
    if x.dim() != 2 or expert_idx.dim() != 2 or expert_idx.shape[0] != x.shape[0]:
        raise B.MoeError("x must be [T, d] and expert_idx [T, k], not %s and %s" % (tuple(x.shape), tuple(expert_idx.shape)))
    B._check_device(x, expert_idx)
    return _Permute.apply(x, expert_idx, E)


class _Combine(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y_perm, expert_scale, inv_perm, active_rows, out_dtype):
        T, k = expert_scale.shape
        inv_perm = inv_perm.clone()                                         # (a layer routes the next batch into the same buffers, through pointers that torch does not see)
        # (rows past y_perm's last are never read, whatever the index says)
        active = None if active_rows is None else active_rows[:1].clamp(max=y_perm.shape[0])
        # (the gate's scales are such a buffer too; where they carry a gradient they are the program's own, and stay in its graph)
        ctx.save_for_backward(y_perm, expert_scale if ctx.needs_input_grad[1] else expert_scale.clone(), inv_perm, active)
        return B.moe_combine(y_perm, inv_perm, expert_scale, T, k, out_dtype=out_dtype, active_rows=active)

    @staticmethod
    def backward(ctx, dout):
        y_perm, expert_scale, inv_perm, active = ctx.saved_tensors
        need = ctx.needs_input_grad[:2]
        call = lambda g, y, s: B.moe_combine_backward(g, y, inv_perm, s, active_rows=active, need=need)  # noqa: E731
        return (*gradient(call, "combine_tokens", whole(dout), y_perm, expert_scale), None, None, None)


def combine_tokens(y_perm, inv_perm, expert_scale, active_rows=None, out_dtype=torch.float32):
    """moe_combine with gradients for y_perm [R, d] and expert_scale fp32 [T, k]: of all tokens (R = T * k), of some of them (rows of others get 0), or of the active rows alone.
    The index, and scales that carry no gradient, may be written again before the backward pass; y_perm may not (torch raises; so it does for a buffer of a layer, of either kind, whose next
    call counts as a change, but where that call is a replay of a captured graph)."""
    if y_perm.dim() != 2 or expert_scale.dim() != 2 or inv_perm.numel() != expert_scale.numel() or (active_rows is not None and active_rows.numel() < 1):
        raise B.MoeError("expert_scale must be [T, k], inv_perm [T * k] and y_perm [R, d], not %s, %s and %s" % tuple(tuple(t.shape) for t in (expert_scale, inv_perm, y_perm)))
    if active_rows is None and y_perm.shape[0] < inv_perm.numel():
        raise B.MoeError("y_perm must have the rows of all %d assignments, or active_rows say how many there are" % inv_perm.numel())
    B._check_device(y_perm, inv_perm, expert_scale, active_rows)
    if not y_perm.is_contiguous() or not expert_scale.is_contiguous():
        y_perm, expert_scale = y_perm.contiguous(), expert_scale.contiguous()
    return _Combine.apply(y_perm, expert_scale, inv_perm, active_rows, out_dtype)
