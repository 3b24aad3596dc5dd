"""Tuning the router of a layer whose experts have been quantised to 4-bit floating point:

    python -m paper_2211_10017_amd.mx4_router_tuning [--steps 60]

The experts stay as they are; the router learns, from the layer's error against what the unquantised layer gave, which experts to use, and
its balance loss keeps their loads even.  The library's part of a step is the gate, the permutation, the expert FFN, the balance loss with the gate scales, and the
gradient of both; the products with the router's weight, the combine as a function of the scales, the error and the optimiser are torch's."""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from .mx4_layer import MoEMx4Layer
from .router import balance_loss


def layer_output(layer, scale):
    """The combine of the last experts() call as a function of the gate scales, for their gradient.  Rows behind the last expert's, those of finished
    sentences, are not written by a call: they count as 0, whatever is in them."""
    row = layer.inv_perm.long()
    y = torch.where((row < layer.expert_offsets[layer.E])[:, None], layer.y_perm.float()[row], 0.0).view(layer.T, layer.k, layer.d)
    return (scale.unsqueeze(-1) * y).sum(1)


def tune(steps=60, T=512, d=256, F=512, E=16, k=2, coef=0.05, lr=0.5, seed=0, report=print):
    """Returns the load of the busiest expert over the mean, before and after, and the losses."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    layer = MoEMx4Layer(T, d, F, E, k)
    for e in range(E):
        layer.load_expert(1, e, torch.randn((d, F), generator=gen, device="cuda") * 0.05)
        layer.load_expert(2, e, torch.randn((F, d), generator=gen, device="cuda") * 0.05)
    wg = torch.randn((d, E), generator=gen, device="cuda") * 0.02
    bias = torch.linspace(0.6, -0.6, E, device="cuda")                      # a router that prefers some experts
    x = torch.randn((T, d), generator=gen, device="cuda").half()
    with torch.no_grad():
        layer.wg.copy_(wg)
        target = layer.forward(x).clone()
    wg, bias = wg.requires_grad_(), bias.requires_grad_()
    optimiser = torch.optim.SGD([wg, bias], lr=lr)
    first = last = None
    losses = []
    for step in range(steps):
        with torch.no_grad():
            layer.wg.copy_(wg)
            layer.gate_bias = bias.detach().clone()
            layer.route(x)
            layer.experts(x)
        logits = x.float() @ wg + bias
        scale, loss, counts, _ = balance_loss(logits, layer.expert_idx, coef, True)
        error = (layer_output(layer, scale) - target).square().mean()
        optimiser.zero_grad()
        (error + loss).backward()
        optimiser.step()
        last = float(counts.max()) / (T * k / E)
        error_now, loss_now = float(error.detach()), float(loss.detach())
        first = last if first is None else first
        losses.append(loss_now)
        if step % 10 == 0 or step + 1 == steps:
            report("step %3d: error %.4f, balance loss %.4f, busiest expert %.2f times the mean load" % (step, error_now, loss_now, last))
    return first, last, losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    B.load()
    tune(ap.parse_args().steps)
