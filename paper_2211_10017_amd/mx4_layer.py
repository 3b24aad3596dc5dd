"""MoEMx4Layer: the expert FFN layer on microscaled 4-bit weights (and 4-bit rows), with MoEExpertLayer's routing: gate, index of the
permutation, expert FFN, un-permute.  Owns the device buffers; forward() only calls the library."""
from __future__ import annotations

import torch

from . import binding as B
from .adapters import LayerIndex


class MoEMx4Layer:
    def __init__(self, T, d, F, E, k, act_dtype=torch.float16, renormalize=True, y_dtype=None, out_dtype=torch.float32, device="cuda:0", activation="relu"):
        # what a whole layer call takes (the gate's limits are the narrowest of the entry points')
        if not (1 <= k <= 2 and k <= E <= B.LAYER_MAX_EXPERTS):
            raise B.MoeError("a layer call takes k = 1 or 2 experts per token and k <= E <= %d experts (k=%d E=%d)"
                             % (B.LAYER_MAX_EXPERTS, k, E))
        if T < 0 or d <= 0 or F <= 0 or d % 64 or F % 64:
            raise B.MoeError("a layer call takes T >= 0 and d, F positive multiples of 64 (T=%d d=%d F=%d)" % (T, d, F))
        if activation not in B.ACTIVATIONS:
            raise B.MoeError("unknown activation %r" % (activation,))
        self.T, self.d, self.F, self.E, self.k, self.renormalize, self.activation = T, d, F, E, k, renormalize, activation
        self.act_dtype = act_dtype
        dev = self.device = torch.device(device)
        R = T * k
        u8, i32 = dict(dtype=torch.uint8, device=dev), dict(dtype=torch.int32, device=dev)
        shapes = B.moe_mx4_shapes
        self.w1, self.w2 = (tuple(torch.empty((E,) + s, **u8) for s in shapes(n, K)) for n, K in ((F, d), (d, F)))      # (codes, scales)
        self.b1 = self.b2 = self.gate_bias = None
        self.adapters = None                                                # LowRankAdapters(E, rank, d, d, act_dtype): an adapter beside each expert
        self.wg = torch.empty((d, E), dtype=act_dtype, device=dev)
        # per-call buffers; y is kept in fp32 for bf16 rows, as in MoEExpertLayer
        self.expert_idx = torch.empty((T, k), **i32)
        self.expert_scale = torch.empty((T, k), dtype=torch.float32, device=dev)
        self.perm_src, self.inv_perm = torch.empty(R, **i32), torch.empty(R, **i32)
        self.expert_offsets = torch.empty(E + 1, **i32)
        self.y_perm = torch.empty((R, d), dtype=y_dtype or (torch.float32 if act_dtype == torch.bfloat16 else act_dtype), device=dev)
        self.out = torch.empty((T, d), dtype=out_dtype, device=dev)
        self.ws_permute = torch.empty(B.moe_permute_workspace_bytes(T, k, E), **u8)
        self.ws_ffn = torch.empty(B.moe_grouped_ffn_mx4_workspace_bytes(T, R, d, F), **u8)

    def load_expert(self, which: int, e: int, w_fp32):
        """Quantise one expert matrix ([d, F] for which = 1, [F, d] for 2) from its fp32 master."""
        codes, scales = self.w1 if which == 1 else self.w2
        B.moe_mx4_quantize_experts(w_fp32.unsqueeze(0), out=(codes[e:e + 1], scales[e:e + 1]))

    def route(self, x, finished=None):
        """Gate and the index of the permutation; finished as for MoEExpertLayer.forward."""
        if x.dtype != self.act_dtype or tuple(x.shape) != (self.T, self.d):
            raise B.MoeError("x must be [T, d] in the layer's activation dtype")
        if finished is not None and finished.numel() != self.T:
            raise B.MoeError("finished must be a contiguous uint8 [T] CUDA tensor")
        B.moe_gate_topk(x, self.wg, self.gate_bias, self.k, self.renormalize, out=(self.expert_idx, self.expert_scale), finished=finished)
        B.moe_permute_index(self.expert_idx, self.E, self.d, x.dtype, self.perm_src, self.inv_perm, self.expert_offsets, self.ws_permute)
        # (written through pointers, here and below: a backward pass that still needs the last call's values raises)
        torch.autograd.graph.increment_version([self.expert_idx, self.expert_scale, self.perm_src, self.inv_perm, self.expert_offsets])

    def experts(self, x):
        """y of every assignment, [T * k, d], in the sorted order of the last route()."""
        B.moe_grouped_ffn_mx4(x, self.expert_offsets, *self.w1, *self.w2, b1=self.b1, b2=self.b2, perm_src=self.perm_src, k=self.k, y_perm=self.y_perm,
                              activation=self.activation, max_rows_per_expert=self.T, workspace=self.ws_ffn)
        if self.adapters is not None:
            self.adapters.add(x, self.y_perm, self.index(), by_assignment=False)
        torch.autograd.graph.increment_version(self.y_perm)
        return self.y_perm

    def index(self):
        """The last route()'s index, as adapters take it; the next one writes it again."""
        return LayerIndex(self.perm_src, self.inv_perm, self.expert_offsets, self.k)

    def forward(self, x, finished=None):
        self.route(x, finished)
        self.experts(x)
        B.moe_combine(self.y_perm, self.inv_perm, self.expert_scale, self.T, self.k, out=self.out, out_dtype=self.out.dtype,
                      active_rows=self.expert_offsets[self.E:])
        torch.autograd.graph.increment_version(self.out)
        return self.out
