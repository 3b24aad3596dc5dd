"""The FFN call against the calls it is made of, bit for bit, through every shape of block that fc1 can have: rows to 4 bits, product in fp32, h to 4 bits, product.
(The products themselves are compared with 64 bits elsewhere.)"""
import numpy as np
import pytest
import torch

from helpers import to_dev
from paper_2211_10017_amd import MoEMx4Layer
from paper_2211_10017_amd import binding as B
from test_gpu_mx4 import DT, repeated_experts, rows_of

pytestmark = pytest.mark.gpu

# fc1's kernel (wavefronts, slabs, lines each; or the row tile's) with h in 4 bits: d, F, rows per expert, types of x that lead there
SHAPES = {"<4, 1, 1": (960, 1088, [1, 3, 0, 2] * 9, ["f16", "bf16", "f32"]), "<4, 1, 1 few blocks": (320, 192, [2, 1, 0, 9], ["f32"]),
          "<8, 1, 1": (1216, 320, [2, 1, 0, 9], ["f32"]), "<8, 1, 1 more blocks": (1152, 3328, [2, 1, 3, 9, 1, 1], ["f16", "bf16"]),
          "<4, 2, 1": (2112, 1088, [1, 2, 1, 1] * 10, ["f16", "bf16", "f32"]), "<2, 2, 2": (1088, 2112, [3, 1] * 40, ["f16", "bf16", "f32"]),
          "<8, 2, 1": (4160, 1088, [1, 2, 1, 1, 33] * 8, ["f16", "bf16", "f32"]), "<2, 2, 1, 2, 3": (1088, 448, [130, 255, 64, 1], ["f16", "bf16", "f32"]),
          "<1, 4, 4, 2, 3": (320, 5568, [700, 1, 645, 830], ["f16", "bf16", "f32"])}


def problem(shape, dtype, bias):
    d, F, rows, _ = SHAPES[shape]
    rng = np.random.default_rng(d + F)
    E, off = len(rows), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R = int(off[-1]) + 3 + (int(off[-1]) + 3) % 2
    src = rng.permutation(R).astype(np.int32)
    x = rows_of(rng, R // 2, d, dtype)
    w1, w2 = ([to_dev(t, torch.uint8) for t in repeated_experts(rng, E, a, b)[:2]] for a, b in ((d, F), (F, d)))
    b1, b2 = [to_dev(rng.standard_normal((E, n)) * 0.5, torch.float16) if bias else None for n in (F, d)]
    return x, to_dev(off, torch.int32), to_dev(src, torch.int32), w1, w2, b1, b2, R


@pytest.mark.parametrize("bias,act,out", [(False, "relu", "f32"), (True, "gelu", "bf16"), (True, "relu", "f16")])
@pytest.mark.parametrize("shape,dtype", [(s, t) for s in SHAPES for t in SHAPES[s][3]])
def test_ffn_is_its_parts(shape, dtype, bias, act, out):
    print(f"mx4 chain {shape} {dtype} bias={bias} {act} {out}", flush=True)
    x, off, src, w1, w2, b1, b2, R = problem(shape, dtype, bias)
    d, F, n = x.shape[1], w1[0].shape[1], int(off[-1])
    y = torch.zeros((R, d), dtype=DT[out], device="cuda:0")
    B.moe_grouped_ffn_mx4(x, off, *w1, *w2, b1=b1, b2=b2, perm_src=src, k=2, y_perm=y, activation=act)
    h = torch.zeros((R, F), device="cuda:0")
    B.moe_grouped_gemm_mx4(*B.moe_mx4_quantize_rows(x), off, *w1, bias=b1, activation=act, perm_src=src, k=2, y=h)
    z = torch.zeros((R, d), dtype=DT[out], device="cuda:0")
    B.moe_grouped_gemm_mx4(*B.moe_mx4_quantize_rows(h), off, *w2, bias=b2, y=z)
    assert torch.isfinite(h).all() and h[:n].any(1).all() and torch.equal(y, z)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_layer_of_no_tokens_and_of_finished_ones_alone(dtype):
    for T in (0, 5):
        layer = MoEMx4Layer(T, 64, 128, 4, 2, act_dtype=DT[dtype])
        for t in (*layer.w1, *layer.w2):
            t.fill_(120)
        layer.wg.zero_()
        layer.out.fill_(7.0)
        layer.y_perm.fill_(torch.nan)                                               # (no call writes the rows of pruned tokens)
        out = layer.forward(torch.ones((T, 64), dtype=DT[dtype], device="cuda:0"), torch.ones(T, dtype=torch.uint8, device="cuda:0"))
        assert out.shape == (T, 64) and not out.any()
