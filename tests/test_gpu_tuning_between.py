"""What happens between a forward pass and its backward pass, and between an optimiser's steps: buffers that layers write again, parameters that others write, gradients as torch may hand
them over."""
import pytest
import torch

from paper_2211_10017_amd import AdamW, LowRankAdapters, MoEExpertLayer, MoEMx4Layer, adapt, combine_tokens, permute_tokens
from paper_2211_10017_amd import binding as B
from paper_2211_10017_amd.adapters import AdapterIndex
from tuning_ref import BF16, F16, F32, generator, routing, sorted_index

pytestmark = pytest.mark.gpu
T, K, D, F, E = 64, 2, 128, 128, 8


def r(gen, *s):
    return torch.randn(s, generator=gen, device="cuda")


def a_layer(kind, gen, k=K):
    layer = MoEMx4Layer(T, D, F, E, k) if kind == "mx4" else MoEExpertLayer(T, D, F, E, k, 4, fuse_routing=False)
    for e in range(E):
        layer.load_expert(1, e, r(gen, D, F) * 0.1)
        layer.load_expert(2, e, r(gen, F, D) * 0.1)
    layer.wg.copy_(r(gen, D, E) * 0.1)
    return layer


@pytest.mark.parametrize("kind", ["mx4", "int4"])
def test_the_scales_of_a_router_that_does_not_learn(kind):
    """The gate's own buffer as it is: the next batch's scales in it change nothing."""
    gen = generator(1)
    layer = a_layer(kind, gen)
    x, other = r(gen, T, D).half(), r(gen, T, D).half()
    adapters = LowRankAdapters(E, 4, D, D, generator=gen)
    adapters.b.normal_(generator=gen)
    adapters.requires_grad_()

    def forward():
        layer.forward(x)
        index = AdapterIndex(layer.perm_src, layer.inv_perm, layer.expert_offsets, K)
        return combine_tokens(adapters(x, layer.y_perm.clone(), index), layer.inv_perm, layer.expert_scale, active_rows=layer.expert_offsets[E:])

    grads = lambda out: torch.autograd.grad(out.square().sum(), adapters.parameters())  # noqa: E731
    want = grads(forward())
    out, scales = forward(), layer.expert_scale.clone()
    layer.forward(other)
    assert not torch.equal(scales, layer.expert_scale)
    assert all(torch.equal(a, b) for a, b in zip(grads(out), want))
