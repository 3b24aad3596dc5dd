"""The operators as they are used together: a layer on 4-bit experts, the tuning of its router, the gradients through torch."""
import numpy as np
import pytest
import torch

from helpers import to_dev
from oracle import mx4
from paper_2211_10017_amd import MoEMx4Layer, balance_loss
from paper_2211_10017_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,F,E,k,dtype,act,finished", [(48, 128, 256, 8, 2, torch.float16, "relu", False), (300, 192, 320, 4, 1, torch.bfloat16, "gelu", True),
                                                         (1, 64, 64, 3, 2, torch.float16, "relu", False)])
def test_layer_is_its_parts(T, d, F, E, k, dtype, act, finished):
    print(f"mx4 layer T={T} d={d} F={F} E={E} k={k}", flush=True)
    rng = np.random.default_rng(T)
    layer = MoEMx4Layer(T, d, F, E, k, act_dtype=dtype, activation=act)
    values = {}
    for which, (K, N) in ((1, (d, F)), (2, (F, d))):
        w = (rng.standard_normal((E, K, N)) * 0.1).astype(np.float32)
        for e in range(E):
            layer.load_expert(which, e, to_dev(w[e], torch.float32))
        values[which] = np.stack([mx4.quantize(w[e].T)[2] for e in range(E)])
    layer.wg.copy_(to_dev(rng.standard_normal((d, E)).astype(np.float32), dtype))
    x = to_dev(rng.standard_normal((T, d)).astype(np.float32), dtype)
    mask = to_dev((rng.random(T) < 0.3).astype(np.uint8), torch.uint8) if finished else None
    out = layer.forward(x, mask).cpu().numpy().astype(np.float64)
    idx, scale = layer.expert_idx.cpu().numpy(), layer.expert_scale.cpu().numpy().astype(np.float64)
    xq = mx4.quantize(x.double().cpu().numpy())[2]
    want = np.zeros((T, d))
    for t in range(T):
        for j in range(k):
            if idx[t, j] < E:
                h = mx4.ACTIVATIONS[act](xq[t:t + 1] @ values[1][idx[t, j]].T)
                want[t] += scale[t, j] * (mx4.quantize(h)[2] @ values[2][idx[t, j]].T)[0]
    # y is rounded to fp16 (bf16 layers keep fp32); an h on the edge between two codes may move a row by a step of one of its F values
    assert np.linalg.norm(out - want) <= 5e-3 * np.linalg.norm(want)
    assert np.abs(out - want).max() <= 0.05 * np.abs(want).max()
    if finished:
        assert not out[mask.cpu().numpy() != 0].any()


def test_layer_refusals():
    for bad in (dict(E=300, k=1), dict(E=8, k=3), dict(E=1, k=2)):
        with pytest.raises(B.MoeError, match="layer call"):
            MoEMx4Layer(16, 64, 128, bad["E"], bad["k"], device="cpu")
    for d, F in ((96, 128), (64, 100)):
        with pytest.raises(B.MoeError, match="multiples of 64"):
            MoEMx4Layer(16, d, F, 8, 1, device="cpu")


@pytest.mark.parametrize("renorm", [True, False])
def test_gradients_through_torch(renorm):
    rng = np.random.default_rng(7)
    z, up = rng.standard_normal((37, 12)).astype(np.float32), rng.standard_normal((37, 2)).astype(np.float32)
    idx = np.argsort(-z, axis=1)[:, :2].astype(np.int32)
    logits = to_dev(z, torch.float32).requires_grad_()
    scale, loss, counts, mean = balance_loss(logits, to_dev(idx, torch.int32), 0.3, renorm)
    assert not counts.requires_grad and not mean.requires_grad
    (2.0 * loss + (scale * to_dev(up, torch.float32)).sum()).backward()
    want = mx4.balance(z, idx, 0.3, renorm, 2.0, up)
    assert np.abs(logits.grad.cpu().numpy() - want["dlogits"]).max() <= 2e-5 * np.abs(want["dlogits"]).max()
    logits.grad = None
    balance_loss(logits, to_dev(idx, torch.int32), 0.3, renorm)[1].backward()                  # the loss alone
    want = mx4.balance(z, idx, 0.3, renorm, 1.0)
    assert np.abs(logits.grad.cpu().numpy() - want["dlogits"]).max() <= 2e-5 * np.abs(want["dlogits"]).max()


def test_router_tuning_evens_the_loads():
    from paper_2211_10017_amd.mx4_router_tuning import tune
    first, last, losses = tune(steps=40, report=lambda line: print(line, flush=True))
    assert losses[-1] < losses[0] and last < first


def test_counted_waits_against_waits_for_everything():
    """The products with every hand-counted wait for a load into LDS replaced by a wait for all of them: the same bits."""
    import ctypes
    from paper_2211_10017_amd.build import LIB_WAITALL
    other = ctypes.CDLL(LIB_WAITALL)
    other.moe_grouped_gemm_mx4.argtypes = B.load().moe_grouped_gemm_mx4.argtypes
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    for rows, K, N in (([3, 0, 17, 32], 704, 96), ([40, 100, 0, 65], 192, 320), ([130, 255, 64, 1], 1088, 352), ([300] * 4, 512, 8192), ([513, 20, 260, 999], 2880, 1056),
                       ([700, 1, 645, 830], 320, 5536), ([2, 1, 9, 0], 1216, 288), ([3, 1, 2, 1] * 10, 2112, 1056), ([3, 1] * 40, 1088, 2080), ([1, 2, 1, 40] * 10, 4160, 1056)):
        print(f"waits {rows} K={K} N={N}", flush=True)
        off = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
        R = int(off[-1])
        a = B.moe_mx4_quantize_rows(torch.randn((R, K), generator=gen, device="cuda"))
        w = B.moe_mx4_quantize_experts(torch.randn((len(rows), K, N), generator=gen, device="cuda"))
        y = B.moe_grouped_gemm_mx4(*a, off, *w, y_dtype=torch.float32)
        z = torch.empty_like(y)
        p = lambda t: t.data_ptr()  # noqa: E731
        rc = other.moe_grouped_gemm_mx4(p(a[0]), p(a[1]), R, None, 1, p(off), R, len(rows), 0, K, N, p(w[0]), p(w[1]), None, -1, p(z), B.MOE_F32, B.current_stream_handle())
        torch.cuda.synchronize()
        assert rc == 0 and torch.equal(y, z)
