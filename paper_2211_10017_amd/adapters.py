"""Low-rank adapters beside a projection: of an expert's rows, or of the requests of a batch (moe_adapters and its backward pass, include/moe_wq.h)."""
from __future__ import annotations

from collections import namedtuple

import torch

from . import binding as B
from .exchange import gradient, whole

class AdapterIndex(namedtuple("AdapterIndex", "perm_src inv_perm offsets k")):
    """The sorted index of rows by adapter (moe_permute): k rows per token."""
    __slots__ = ()
    by_assignment = property(lambda self: self.k == 1)      # how y lies unless a call says so: one row per request, in the requests' order


class LayerIndex(AdapterIndex):
    """An expert layer's: y is sorted by expert, also with one expert per token."""
    __slots__ = ()
    by_assignment = False


def adapter_index(adapter_idx, E: int):
    """Index of requests: adapter_idx int32 [T] on the device, E for a request without an adapter (E <= 1024, moe_permute's limit).  Worth keeping while the batch is the same."""
    B._check_device(adapter_idx)
    T, dev = adapter_idx.numel(), adapter_idx.device
    index = AdapterIndex(*(torch.empty(n, dtype=torch.int32, device=dev) for n in (T, T, E + 1)), 1)
    workspace = torch.empty(B.moe_permute_workspace_bytes(T, 1, E), dtype=torch.uint8, device=dev)
    B.moe_permute_index(adapter_idx.view(T, 1), E, 8, torch.float16, index.perm_src, index.inv_perm, index.offsets, workspace)
    return index


class _Adapt(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, a, b, scale, index, by_assignment, y_dtype):
        R, rank = index.perm_src.numel(), a.shape[1]
        v = torch.empty(R, rank, dtype=torch.float32, device=x.device)
        # (copies: a layer routes the next batch into the same buffers, through pointers that torch does not see)
        perm_src, inv_perm, offsets = (t.clone() for t in index[:3])
        out = B.moe_adapters(x, a, b, offsets, perm_src, index.k, scale, by_assignment, y=y, y_dtype=y_dtype, v=v)
        ctx.save_for_backward(x, a, b, scale, v, perm_src, inv_perm, offsets)
        ctx.k, ctx.by_assignment, ctx.tokens = index.k, by_assignment, x.shape[0]
        return out

    @staticmethod
    def backward(ctx, dout):
        x, a, b, scale, v, perm_src, inv_perm, offsets = ctx.saved_tensors
        need_x, need_y, need_a, need_b = ctx.needs_input_grad[:4]

        def call(dout, x, a, b):
            dx, da, db = B.moe_adapters_backward(dout, x, a, b, v, offsets, perm_src, ctx.k, scale, ctx.by_assignment, need=(need_x, need_a, need_b))
            if need_x and not (ctx.by_assignment and ctx.k == 1):          # (a token's rows in one: those of no adapter are 0)
                order = torch.arange(dx.shape[0], dtype=torch.int32, device=dx.device) if ctx.by_assignment else inv_perm
                dx = B.moe_permute_backward(dx, order, ctx.tokens, ctx.k)
            return dx, da, db

        dx = da = db = None
        if need_x or need_a or need_b:
            rows = dout if dout.stride(-1) == 1 and dout.stride(0) % 8 == 0 and dout.stride(0) >= dout.shape[1] and dout.data_ptr() % 16 == 0 else whole(dout)
            dx, da, db = gradient(call, "adapt", rows, x, a, b)
        return dx, dout if need_y else None, da, db, None, None, None, None


def adapt(x, y, a, b, index, scale=None, by_assignment: bool = False, y_dtype=None):
    """moe_adapters as a function with gradients for x [T, K], y, a [E, rank, K] and b [E, rank, N]: y[r] + scale[e] * (A[e] x[t]) B[e], in a tensor of its own (y None: the second term).
    The index may be written again before the backward pass; the others may not.  scale takes no gradient.  x's gradient is rounded to its type row by row, before a token's are added."""
    if scale is not None and scale.requires_grad:
        raise B.MoeError("an adapter's scale takes no gradient")
    return _Adapt.apply(x, y, a, b, scale, index, by_assignment, y_dtype)


class LowRankAdapters:
    """E adapters from K to N channels (index() makes one of up to 1024, moe_permute's limit; a caller's own serves up to 4096).  a starts as normal numbers, b as 0: an adapter begins by
    changing nothing."""

    def __init__(self, E, rank, K, N, dtype=torch.float16, alpha=None, device="cuda:0", generator=None):
        if not (1 <= E <= 4096 and 1 <= rank <= 128) or K <= 0 or N <= 0 or K % 8 or N % 8:
            raise B.MoeError("adapters take 1 <= E <= 4096, 1 <= rank <= 128 and K, N positive multiples of 8 (E=%d rank=%d K=%d N=%d)" % (E, rank, K, N))
        if dtype not in (torch.float16, torch.bfloat16):
            raise B.MoeError("adapters are fp16 or bf16")
        self.E, self.rank, self.K, self.N = E, rank, K, N
        self.a = (torch.randn((E, rank, K), device=device, generator=generator) * K ** -0.5).to(dtype)
        self.b = torch.zeros((E, rank, N), dtype=dtype, device=device)
        self.scale = torch.full((E,), (rank if alpha is None else alpha) / rank, dtype=torch.float32, device=device)

    def parameters(self):
        return [self.a, self.b]

    def requires_grad_(self, flag: bool = True):
        for t in self.parameters():
            t.requires_grad_(flag)
        return self

    def index(self, adapter_idx):
        return adapter_index(adapter_idx, self.E)

    def add(self, x, y, index, by_assignment=None):
        """y += the adapters' term, in place, without gradients (for autograd y has been changed).  Requests (k = 1): y in their order; an expert layer's rows (its index()): sorted."""
        B.moe_adapters(x, self.a.detach(), self.b.detach(), index.offsets, index.perm_src, index.k, self.scale, index.by_assignment if by_assignment is None else by_assignment, y=y, out=y)
        torch.autograd.graph.increment_version(y)
        return y

    def __call__(self, x, y, index, by_assignment=None):
        return adapt(x, y, self.a, self.b, index, self.scale, index.by_assignment if by_assignment is None else by_assignment)
