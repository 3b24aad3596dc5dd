"""balance_loss through torch's autograd on a layer's own buffers."""
import numpy as np
import pytest
import torch

from helpers import to_dev
from oracle import mx4
from paper_2211_10017_amd import MoEMx4Layer, balance_loss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("renorm", [True, False])
def test_two_batches_routed_before_their_backward(renorm):
    rng = np.random.default_rng(21)
    layer = MoEMx4Layer(40, 64, 64, 8, 2, renormalize=renorm)
    layer.wg.copy_(to_dev(rng.standard_normal((64, 8)) * 0.2, torch.float16))
    wg = layer.wg.float()
    total, kept = 0.0, []
    for _ in range(2):                                                             # gradients of two batches accumulate
        x = to_dev(rng.standard_normal((40, 64)), torch.float16)
        layer.route(x)
        logits = (x.float() @ wg).requires_grad_()
        up = rng.standard_normal((40, 2)).astype(np.float32)
        scale, loss, _, _ = balance_loss(logits, layer.expert_idx, 0.3, renorm)
        total = total + 2.0 * loss + (scale * to_dev(up, torch.float32)).sum()
        kept.append((logits, layer.expert_idx.cpu().numpy().copy(), up))
    assert (kept[0][1] != kept[1][1]).any()
    total.backward()
    for logits, idx, up in kept:
        want = mx4.balance(logits.detach().cpu().numpy(), idx, 0.3, renorm, 2.0, up)["dlogits"]
        assert np.abs(logits.grad.cpu().numpy() - want).max() <= 2e-5 * np.abs(want).max()


def test_a_loss_and_a_statistic_changed_in_place():
    rng = np.random.default_rng(22)
    z = rng.standard_normal((37, 12)).astype(np.float32)
    idx = np.argsort(-z, axis=1)[:, :2].astype(np.int32)
    logits = to_dev(z, torch.float32).requires_grad_()
    _, loss, _, mean = balance_loss(logits, to_dev(idx, torch.int32), 0.3, True)
    mean.mul_(0.9)                                                                 # a moving average
    loss += 7.0
    loss.backward()
    want = mx4.balance(z, idx, 0.3, True, 1.0)
    assert abs(float(loss.detach()) - 7.0 - want["loss"]) <= 1e-5
    assert np.abs(logits.grad.cpu().numpy() - want["dlogits"]).max() <= 2e-5 * np.abs(want["dlogits"]).max()
