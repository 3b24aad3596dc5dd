"""The FFN's calls whose fc1 quantises its rows for itself, and the streamed products' numbers that are none."""
import numpy as np
import pytest
import torch

from helpers import to_dev
from oracle import mx4
from paper_2211_10017_amd import binding as B
from test_gpu_mx4 import DT, ROUND, TINY, experts_of, ffn_with_bounds, held, host, repeated_experts, rows_of

pytestmark = pytest.mark.gpu

# rows per expert, at most 24 on average: one, none, sixteen, more than an item holds
LOADS = {"one": [0, 1], "few": [3, 0, 0, 7, 1, 0], "full": [24, 22], "uneven": [33, 2, 1, 0, 16, 65, 3], "many": [1] * 70 + [0] * 7 + [2, 5]}
# (load, d, F): fc1 by four wavefronts up to d = 1024, by eight beyond; whole and half groups of scales, one chunk of K and several passes of them
SIZES = [("one", 64, 64), ("few", 192, 320), ("full", 704, 576), ("uneven", 1024, 1024), ("many", 512, 192), ("one", 1088, 4096), ("few", 2112, 1088), ("full", 4160, 256),
         ("uneven", 1216, 64), ("many", 2880, 64)]


def batch(load, seed):
    rng = np.random.default_rng(seed)
    rows = LOADS[load]
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R = int(off[-1]) + 1                                                            # the last row, or the last two, belong to a pruned token
    R += R % 2
    return rng, len(rows), off, R, R // 2, rng.permutation(R).astype(np.int32)


def all_kinds(rng, T, d, dtype):
    """Rows of blocks of every kind, and rows of the type's smallest numbers, subnormal ones among them, of zeros, of the largest, with a NaN and with infinities."""
    x = rows_of(rng, T, d, dtype)
    low = torch.finfo(DT[dtype])
    for t in range(T):
        kind = t % 12
        if kind == 1: x[t] = to_dev(rng.integers(-40, 41, d) * low.smallest_normal * 2.0 ** -4, DT[dtype])          # noqa: E701
        elif kind == 2: x[t] = to_dev(rng.integers(-3, 4, d) * low.smallest_normal * low.eps, DT[dtype])            # noqa: E701  (the last bits there are)
        elif kind == 4: x[t] = 0.0                                                                                  # noqa: E701
        elif kind == 6: x[t] = to_dev(rng.uniform(-1, 1, d) * low.max, DT[dtype])                                    # noqa: E701
        elif kind == 8: x[t, int(rng.integers(d))] = torch.nan                                                       # noqa: E701
        elif kind == 9: x[t, int(rng.integers(d))] = torch.inf                                                       # noqa: E701
        elif kind == 10: x[t, d - 1] = -torch.inf                                                                    # noqa: E701
    return x


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("load,d,F", SIZES)
def test_the_same_bits_as_quantised_rows(load, d, F, dtype):
    """fc1 on rows that it quantises itself and on those that the quantiser has quantised: y bit for bit, through weights that bring the smallest rows' h up into range."""
    rng, E, off, R, T, src = batch(load, d + F)
    print(f"mx4 fused {load} d={d} F={F} {dtype}", flush=True)
    x = all_kinds(rng, T, d, dtype)
    w1, w2 = ([to_dev(t, torch.uint8) for t in repeated_experts(rng, E, a, b)[:2]] for a, b in ((d, F), (F, d)))
    if dtype == "bf16":
        w1[1] += 60                                                                 # 2^60 times the size: the smallest rows are 2^-133
    off, src = to_dev(off, torch.int32), to_dev(src, torch.int32)
    y = torch.zeros((R, d), device="cuda:0")
    B.moe_grouped_ffn_mx4(x, off, *w1, *w2, perm_src=src, k=2, y_perm=y)
    h = torch.zeros((R, F), device="cuda:0")
    B.moe_grouped_gemm_mx4(*B.moe_mx4_quantize_rows(x), off, *w1, activation="relu", perm_src=src, k=2, y=h)
    z = torch.zeros((R, d), device="cuda:0")
    B.moe_grouped_gemm_mx4(*B.moe_mx4_quantize_rows(h), off, *w2, y=z)
    n = int(off[-1])
    assert torch.equal(torch.isnan(y), torch.isnan(z)) and torch.equal(torch.nan_to_num(y), torch.nan_to_num(z))
    bad = (~torch.isfinite(x.float()).all(1))[(src[:n] // 2).long()]
    kind = (src[:n] // 2) % 12
    sure = torch.ones_like(bad) if dtype == "f16" else kind != 6                    # (bf16: the largest rows times 2^60 pass what 32 bits hold)
    assert torch.equal(torch.isnan(y[:n])[sure], bad[:, None].expand(n, d)[sure])   # a row that holds a NaN or an infinity, and no other
    if T > 24:                                                                      # (the smallest bf16 number is 0 in units of the smallest scale)
        assert y[:n][kind == 1].any() and (dtype == "bf16" or y[:n][kind == 2].any())


@pytest.mark.parametrize("dtype,bias,act", [("f16", True, "gelu"), ("bf16", False, "relu"), ("bf16", True, "gelu")])
@pytest.mark.parametrize("load,d,F", SIZES)
def test_against_64_bits(load, d, F, dtype, bias, act):
    rng, E, off, R, T, src = batch(load, d)
    print(f"mx4 fused ffn {load} d={d} F={F} {dtype} bias={bias} {act}", flush=True)
    x = rows_of(rng, T, d, dtype)
    w1, w2 = experts_of(rng, E, d, F), experts_of(rng, E, F, d)
    b1, b2 = [(rng.standard_normal((E, n)) * 0.1).astype(np.float16) if bias else None for n in (F, d)]
    f = lambda t, dt: None if t is None else to_dev(t, dt)  # noqa: E731
    y = torch.full((R, d), -77.0, dtype=DT[dtype], device="cuda:0")
    B.moe_grouped_ffn_mx4(x, f(off, torch.int32), f(w1[0], torch.uint8), f(w1[1], torch.uint8), f(w2[0], torch.uint8), f(w2[1], torch.uint8), b1=f(b1, torch.float16),
                          b2=f(b2, torch.float16), perm_src=f(src, torch.int32), k=2, y_perm=y, activation=act)
    got, n = host(y.double()), off[-1]
    assert (got[n:] == -77.0).all()
    wide = lambda t: None if t is None else t.astype(np.float64)  # noqa: E731
    want, size, moved, _ = ffn_with_bounds(host(x.double()), off, src // 2, w1[2], w2[2], wide(b1), wide(b2), act)
    tol = 1.13 * (F / 64 + 9) * 2.0 ** -23 * size[:n] + moved[:n]
    assert (np.abs(got[:n] - want[:n]) <= tol + ROUND[dtype] * (np.abs(want[:n]) + tol) + TINY[dtype]).all()


@pytest.mark.parametrize("K,N,rows", [(256, 64, [20, 25]), (1216, 96, [3, 9]), (2112, 1056, [1, 2, 1, 1] * 10), (1088, 2080, [3, 1] * 40)])
def test_streamed_product_of_blocks_that_are_not_numbers(K, N, rows):
    """A NaN scale of a row spoils that row alone, of a channel that channel alone; rows of zeros give zeros."""
    rng = np.random.default_rng(K)
    E, off = len(rows), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R = int(off[-1])
    a, w = held(rng, R, K), [t.copy() for t in repeated_experts(rng, E, K, N)[:2]]
    last = K // 32 - 1
    a[1][last // 4, 1, last % 4] = 255                                              # (the last block there is)
    a[0][3] = 0
    w[1][0, 0, 9, 1] = w[1][E - 1, last // 4, N - 1, last % 4] = 255
    y = host(B.moe_grouped_gemm_mx4(*[to_dev(t, torch.uint8) for t in a[:2]], to_dev(off, torch.int32), *[to_dev(t, torch.uint8) for t in w], y_dtype=torch.float32))
    bad = np.zeros((R, N), dtype=bool)
    bad[1] = True
    bad[:off[1], 9] = bad[off[E - 1]:, N - 1] = True
    assert (np.isnan(y) == bad).all() and not y[3, ~bad[3]].any()


@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_streamed_activations_keep_what_is_not_a_number(act, dtype):
    rng = np.random.default_rng(12)
    x = to_dev(rng.standard_normal((20, 128)), DT[dtype])
    x[3, 5], x[16, 100] = torch.nan, -torch.inf
    w1, w2 = [[to_dev(t, torch.uint8) for t in experts_of(rng, 1, a, b)[:2]] for a, b in ((128, 64), (64, 128))]
    off = to_dev(np.array([0, 20]), torch.int32)
    bad = torch.zeros(20, dtype=torch.bool, device="cuda:0")
    bad[3] = bad[16] = True
    y = B.moe_grouped_ffn_mx4(x, off, *w1, *w2, activation=act)
    assert torch.equal(torch.isnan(y), bad[:, None].expand_as(y))
