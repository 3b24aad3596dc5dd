"""AdamW over many tensors, forty in a launch, states in 32 or 8 bits (moe_adamw, include/moe_wq.h)."""
from __future__ import annotations

import torch

from . import binding as B

_HALVES = (torch.float16, torch.bfloat16)


class AdamW:
    """16-bit parameters are kept in fp32 beside themselves (`masters`) and written as copies of that in the same pass; what others write into one between
    two steps (not through .data, which torch does not count) goes into its master.  step() takes the gradients that are there; a parameter without one stays as it is, and its steps are counted
    from its own first one on (`counts`).  States in 8 bits are rounded up or down by chance, the same in every run: to the nearest number they could not follow their averages."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, bits=32):
        self.params = list(params)
        if bits not in (8, 32):
            raise B.MoeError("states have 8 or 32 bits")
        if not self.params or any(p.dtype not in _HALVES + (torch.float32,) or not p.is_contiguous() for p in self.params):
            raise B.MoeError("parameters must be contiguous tensors of fp16, bf16 or fp32")
        if len({p.data_ptr() for p in self.params if p.numel()}) < sum(p.numel() > 0 for p in self.params):
            raise B.MoeError("a parameter is in the list twice")
        self.lr, self.betas, self.eps, self.weight_decay, self.bits = lr, tuple(betas), eps, weight_decay, bits
        self.counts = [0] * len(self.params)                # steps that each parameter has taken: its moments begin at 0, whenever that is
        self.masters = [p.detach().float() if p.dtype in _HALVES else None for p in self.params]
        self._seen = [None if p.is_inference() else p._version for p in self.params]        # as the masters know them (inference tensors have no version)

        def state(p):
            if bits == 32:
                return torch.zeros(p.numel(), dtype=torch.float32, device=p.device)
            return tuple(torch.zeros(n, dtype=torch.uint8, device=p.device) for n in (p.numel(), (p.numel() + 31) // 32))

        self.exp_avg, self.exp_avg_sq = ([state(p) for p in self.params] for _ in range(2))

    @property
    def steps(self):
        """The most steps that a parameter has taken."""
        return max(self.counts)

    @steps.setter
    def steps(self, number):
        self.counts[:] = [int(number)] * len(self.params)

    def step(self, grad_scale: float = 1.0):
        if self.params[0].device.type == "cuda" and torch.cuda.is_current_stream_capturing():
            raise B.MoeError("a captured step would have the same number in every replay: capture moe_adamw, with the step's number on the device")
        groups = {}
        for i, (p, master, count) in enumerate(zip(self.params, self.masters, self.counts)):
            g = p.grad
            if g is not None:
                if g.is_sparse:
                    raise B.MoeError("gradients must be dense")
                key = None if master is None else p.dtype, g.dtype, count + 1
                if key not in groups:
                    groups[key] = [], [], []
                for to, what in zip(groups[key], (i, p, g.contiguous())):
                    to.append(what)
        lib, calls = B.load(), []
        for (half, _, number), (at, params, grads) in groups.items():
            masters = [self.masters[i] for i in at] if half else None
            call = B.adamw_arguments(masters or params, grads, [self.exp_avg[i] for i in at], [self.exp_avg_sq[i] for i in at], number, self.lr, self.betas, self.eps, self.weight_decay, grad_scale,
                                     params if half else None, "random")
            calls.append((at, params, number, half, *call))
        # (a refusal leaves everything as it was, so all calls are checked before the first is made; one alone is by itself)
        if len(calls) > 1:
            for call in calls:
                B._check(lib.moe_adamw_check(*call[4]), "moe_adamw")
        for at, params, number, half, arguments, _ in calls:
            if half:
                for i, p in zip(at, params):
                    if not p.is_inference() and p._version != self._seen[i]:
                        self._take_over(i)
            B._check(lib.moe_adamw(*arguments, B._stream()), "moe_adamw")
            # (written through pointers: a backward pass that still needs the old values raises)
            torch.autograd.graph.increment_version(params)
            for i in at:
                self.counts[i] = number
            if half:
                for i, p in zip(at, params):
                    self._seen[i] = None if p.is_inference() else p._version

    def _take_over(self, i):
        """A parameter's new values into its master; where the parameter is still the master's rounding, the master stays."""
        master, p = self.masters[i], self.params[i].detach()
        master.copy_(torch.where(master.to(p.dtype) == p, master, p.float()))

    def zero_grad(self, set_to_none: bool = True):
        for p in self.params:
            if p.grad is not None:
                if set_to_none:
                    p.grad = None
                else:
                    p.grad.zero_()

    def state_dict(self):
        """The optimiser's own tensors and counts, which later steps change: to keep them, copy or save them."""
        return dict(steps=self.counts, bits=self.bits, masters=self.masters, exp_avg=self.exp_avg, exp_avg_sq=self.exp_avg_sq)

    def load_state_dict(self, state):
        if state["bits"] != self.bits or len(state["exp_avg"]) != len(self.params):
            raise B.MoeError("the state belongs to other parameters, or has other bits")
        flat = lambda s: [t for x in s for t in (x if isinstance(x, tuple) else (x,)) if t is not None]  # noqa: E731
        mine, theirs = (flat(s["masters"]) + flat(s["exp_avg"]) + flat(s["exp_avg_sq"]) for s in (self.state_dict(), state))
        steps = [state["steps"]] * len(self.params) if isinstance(state["steps"], int) else list(state["steps"])      # (one number: a state of one count for all)
        if len(steps) != len(self.params) or [t.shape for t in mine] != [t.shape for t in theirs]:
            raise B.MoeError("the state belongs to other parameters")
        for m, t in zip(mine, theirs):
            m.copy_(t)
        self.counts[:] = steps
