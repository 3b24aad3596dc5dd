"""The microscaled 4-bit operators against 64 bits: codes, scales and values bit for bit; products within what 32-bit sums and the output's own rounding
can be away; the FFN with, on top, what an h on the edge between two codes can move."""
import numpy as np
import pytest
import torch

from helpers import to_dev
from oracle import mx4
from paper_2211_10017_amd import binding as B

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -133, "f32": 2.0 ** -149}


def host(t):
    return t.cpu().numpy()


def rows_of(rng, R, K, dtype):
    """Rows with blocks of every kind: ordinary, tiny, large, zero, on the halfway points of the codes, single spikes."""
    x = rng.standard_normal((R, K)) * np.exp(rng.standard_normal(K))
    b = x.reshape(R, -1, 32)
    kind = rng.integers(0, 8, b.shape[:2])
    b[kind == 1] = 0.0
    b[kind == 2] *= 2.0 ** -13
    b[kind == 3] = rng.choice(np.concatenate([mx4.GRID, (mx4.GRID[1:] + mx4.GRID[:-1]) / 2, [7.0, -7.5, -0.0]]), b[kind == 3].shape) * 0.25
    b[kind == 4, 5] = 900.0
    return to_dev(x, DT[dtype])


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 64), (3, 128), (16, 192), (17, 320), (5, 2880), (64, 1024), (1000, 704), (4097, 512)])
def test_rows_bit_exact(R, K, dtype):
    print(f"mx4 rows R={R} K={K} {dtype}", flush=True)
    x = rows_of(np.random.default_rng(R + K), R, K, dtype)
    codes, scales = B.moe_mx4_quantize_rows(x)
    want_codes, want_scales, want = mx4.quantize(host(x.double()))
    assert (host(codes) == want_codes).all() and (host(scales) == want_scales).all()
    for name in DT:
        got = host(B.moe_mx4_dequantize(codes, scales, DT[name]).double())
        assert (got == host(torch.from_numpy(want).to(DT[name]).double())).all(), name


def test_rows_at_the_ends_of_the_range():
    """fp32: subnormal numbers, the smallest and largest scales, infinities and NaN, each in a block of its own."""
    rng = np.random.default_rng(3)
    tops = [2.0 ** -149, 3 * 2.0 ** -149, 2.0 ** -127, 2.0 ** -126, 1.75 * 2.0 ** -126, 2.0 ** -125, 2.0 ** -124, 2.0 ** 126, np.finfo(np.float32).max, 65504.0, np.inf, -np.inf, np.nan]
    v = np.zeros((2, 32 * 14), dtype=np.float32)
    for i, t in enumerate(tops):
        with np.errstate(all="ignore"):
            v[:, 32 * i:32 * i + 32] = (rng.uniform(-1, 1, (2, 32)) * (1.0 if not np.isfinite(t) else t)).astype(np.float32)
        v[:, 32 * i + 7] = t
    codes, scales = B.moe_mx4_quantize_rows(to_dev(v, torch.float32))
    want_codes, want_scales, want = mx4.quantize(v)
    assert (host(scales) == want_scales).all()
    assert (host(codes) == want_codes).all()
    got = host(B.moe_mx4_dequantize(codes, scales, torch.float32)).astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and (got[~np.isnan(got)] == want[~np.isnan(want)].astype(np.float32)).all()


def test_strided_rows_on_another_stream():
    rng = np.random.default_rng(5)
    wide = to_dev(rng.standard_normal((33, 512)), torch.bfloat16)
    part = wide[:, 128:320]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        codes, scales = B.moe_mx4_quantize_rows(part)
    side.synchronize()
    want_codes, want_scales, _ = mx4.quantize(host(part.double()))
    assert (host(codes) == want_codes).all() and (host(scales) == want_scales).all()


@pytest.mark.parametrize("E,K,N", [(1, 64, 32), (3, 192, 96), (2, 1024, 256), (1, 2880, 288), (5, 128, 1056)])
def test_experts_bit_exact(E, K, N):
    print(f"mx4 experts E={E} K={K} N={N}", flush=True)
    rng = np.random.default_rng(E + K)
    w = np.ascontiguousarray(np.stack([host(rows_of(rng, N, K, "f32")).T for _ in range(E)]))
    codes, scales = B.moe_mx4_quantize_experts(to_dev(w, torch.float32))
    values = host(B.moe_mx4_dequantize(codes, scales, torch.float32)).astype(np.float64)
    for e in range(E):
        want_codes, want_scales, want = mx4.quantize(w[e].T)
        assert (host(codes[e]) == want_codes).all() and (host(scales[e]) == want_scales).all() and (values[e] == want).all()
    one = B.moe_mx4_quantize_experts(to_dev(w[E - 1:], torch.float32))           # an expert alone gives the same bytes
    assert torch.equal(one[0][0], codes[-1]) and torch.equal(one[1][0], scales[-1])


def held(rng, shape_rows, K, size=1.0):
    """Rows in the 4-bit format with their values, and junk in the scale bytes of blocks past K."""
    codes, scales, values = mx4.quantize(rng.standard_normal((shape_rows, K)) * np.exp(0.5 * rng.standard_normal(K)) * size)
    last = K // 32 - 4 * (scales.shape[0] - 1)
    scales[-1, :, last:] = 255
    return codes, scales, values


def experts_of(rng, E, K, N):
    parts = [held(rng, N, K, 0.02) for _ in range(E)]
    return tuple(np.stack([p[i] for p in parts]) for i in range(3))


# rows per expert: one, none, odd numbers, the edges of 16, 32, 64, 128 and 256 rows, everything in one expert
LOADS = {"one": [0, 1], "few": [3, 0, 0, 7, 1, 0], "edges": [15, 16, 17, 31, 32, 33], "tiles": [63, 65, 0, 64, 127, 129], "tall": [0, 255, 257], "lone": [700],
         "many": [1] * 70 + [0] * 7 + [2, 5]}
FFN_LOADS = dict(LOADS, large=[700, 1, 645, 830])

@pytest.mark.parametrize("load", LOADS)
@pytest.mark.parametrize("K,N,out,bias,act", [(64, 32, "f32", False, None), (192, 96, "f16", True, "relu"), (1024, 256, "f32", True, None), (2880, 320, "bf16", False, "gelu"),
                                              (576, 544, "f32", True, "relu")])
def test_product(load, K, N, out, bias, act):
    print(f"mx4 product {load} K={K} N={N} {out} bias={bias} act={act}", flush=True)
    rng = np.random.default_rng(K + N)
    rows = LOADS[load]
    E, pruned, k = len(rows), 3, 2
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R, T = int(off[-1]) + pruned, int(off[-1]) + 5
    src = rng.integers(0, T * k, R).astype(np.int32)
    a, w = held(rng, T, K), experts_of(rng, E, K, N)
    b = (rng.standard_normal((E, N)) * 0.5).astype(np.float16) if bias else None
    y = torch.full((R, N), -77.0, dtype=DT[out], device="cuda:0")
    B.moe_grouped_gemm_mx4(to_dev(a[0], torch.uint8), to_dev(a[1], torch.uint8), to_dev(off, torch.int32), to_dev(w[0], torch.uint8), to_dev(w[1], torch.uint8),
                           bias=None if b is None else to_dev(b, torch.float16), activation=act, perm_src=to_dev(src, torch.int32), k=k, y=y)
    got = host(y.double())
    assert (got[off[-1]:] == -77.0).all()                                           # rows of no expert stay as they were
    v, size = mx4.product(a[2][src // k], off, w[2], None if b is None else b.astype(np.float64))
    check_rows(got[:off[-1]], mx4.ACTIVATIONS[act](v[:off[-1]]), size[:off[-1]], K, out, act)


def check_rows(got, want, size, K, out, act):
    # K/64 matrix instructions in a chain and up to eight partial sums of it, each addition off by at most 2^-23 of the terms' magnitudes so far; activations pass an
    # error on at most 1.13 times and GELU adds 4e-7 |v| of its own; the result is rounded once
    tol = 1.13 * (K / 64 + 9) * 2.0 ** -23 * size + (4e-7 * (np.abs(want) + size) if act == "gelu" else 0)
    assert (np.abs(got - want) <= tol + ROUND[out] * (np.abs(want) + tol) + TINY[out]).all(), np.abs(got - want).max()


def repeated_experts(rng, E, K, N, different=2):
    """E experts of `different` kinds (codes at random, so cheap to make in 64 bits): codes, scales, and the values of each kind."""
    codes = rng.integers(0, 256, (different, N, K // 2)).astype(np.uint8)
    scales = rng.integers(118, 123, (different, -(-K // 128), N, 4)).astype(np.uint8)
    kind = np.arange(E) % different
    return codes[kind], scales[kind], [mx4.dequantize(codes[i], scales[i]) for i in kind[:different]]


# every shape of block, by what leads to it
SHAPES = {"large tiles": (320, 5536, [700, 1, 645, 830]), "large tiles, one odd half group": (192, 5472, [609, 33, 97, 1000, 545]),      # (rows of the last tile: one to four times 32)
          "small tiles": (1088, 416, [130, 255, 64, 1]), "streamed, one slab, short K": (960, 1056, [1, 3, 0, 2] * 9),
          "streamed, one slab": (1216, 288, [2, 1, 0, 9]), "streamed, two slabs": (2112, 1056, [1, 2, 1, 1] * 10), "streamed, two lines each": (1088, 2080, [3, 1] * 40),
          "streamed, long K": (4160, 1056, [1, 2, 1, 1, 33] * 8)}


@pytest.mark.parametrize("out", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes_of_blocks(shape, out):
    K, N, rows = SHAPES[shape]
    print(f"mx4 product {shape} K={K} N={N} {out}", flush=True)
    rng = np.random.default_rng(K)
    E, off = len(rows), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    a, w = held(rng, int(off[-1]), K), repeated_experts(rng, E, K, N)
    src = rng.permutation(int(off[-1])).astype(np.int32)
    y = B.moe_grouped_gemm_mx4(*[to_dev(t, torch.uint8) for t in a[:2]], to_dev(off, torch.int32), *[to_dev(t, torch.uint8) for t in w[:2]], perm_src=to_dev(src, torch.int32),
                               y_dtype=DT[out])
    got, v = host(y.double()), a[2][src]
    for e in range(E):
        r = slice(off[e], off[e + 1])
        check_rows(got[r], v[r] @ w[2][e % 2].T, np.abs(v[r]) @ np.abs(w[2][e % 2]).T, K, out, None)


def test_a_bound_on_the_rows_of_an_expert_only_chooses():
    """A buffer of many rows of which few are in use: with and without the caller's bound on them, and with one that does not hold, the same product."""
    rng = np.random.default_rng(8)
    off = np.array([0, 3, 5, 41], dtype=np.int32)
    a, w = held(rng, 200, 576), experts_of(rng, 3, 576, 96)
    args = [to_dev(t, torch.uint8) for t in a[:2]] + [to_dev(off, torch.int32)] + [to_dev(t, torch.uint8) for t in w[:2]]
    want, size = mx4.product(a[2], off, w[2])
    for most in (0, 1, 36, 200, 2 ** 31 - 1):
        y = torch.full((200, 96), -77.0, device="cuda:0")
        got = host(B.moe_grouped_gemm_mx4(*args, y=y, max_rows_per_expert=most).double())
        assert (got[41:] == -77.0).all()
        check_rows(got[:41], want[:41], size[:41], 576, "f32", None)


def test_product_without_an_index_and_its_repeats():
    rng = np.random.default_rng(9)
    rows = [40, 0, 90, 3]
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    a, w = held(rng, int(off[-1]), 512), experts_of(rng, 4, 512, 128)
    args = [to_dev(t, torch.uint8) for t in a[:2]] + [to_dev(off, torch.int32)] + [to_dev(t, torch.uint8) for t in w[:2]]
    y = B.moe_grouped_gemm_mx4(*args, y_dtype=torch.float32)
    check_rows(host(y.double()), *mx4.product(a[2], off, w[2]), 512, "f32", None)
    for _ in range(3):
        assert torch.equal(B.moe_grouped_gemm_mx4(*args, y_dtype=torch.float32), y)


def test_product_of_blocks_that_are_not_numbers():
    """A NaN scale of a row spoils that row alone, of a channel that channel alone; rows of zeros give zeros."""
    rng = np.random.default_rng(11)
    K, N, rows = 256, 64, [20, 40]
    off = np.array([0, 20, 60], dtype=np.int32)
    a, w = held(rng, 60, K), experts_of(rng, 2, K, N)
    a[1][1, 25, 2] = 255
    a[0][7] = 0
    w[1][0, 0, 9, 1] = 255
    y = host(B.moe_grouped_gemm_mx4(*[to_dev(t, torch.uint8) for t in a[:2]], to_dev(off, torch.int32), *[to_dev(t, torch.uint8) for t in w[:2]], y_dtype=torch.float32))
    bad = np.zeros((60, N), dtype=bool)
    bad[25] = True
    bad[:20, 9] = True
    assert (np.isnan(y) == bad).all() and not y[7, ~bad[7]].any()


@pytest.mark.parametrize("act", ["relu", "gelu"])
def test_activations_keep_what_is_not_a_number(act):
    rng = np.random.default_rng(12)
    x = to_dev(rng.standard_normal((70, 128)), torch.bfloat16)
    x[3, 5], x[66, 100] = torch.nan, -torch.inf
    w1, w2 = [[to_dev(t, torch.uint8) for t in experts_of(rng, 1, a, b)[:2]] for a, b in ((128, 64), (64, 128))]
    off = to_dev(np.array([0, 70]), torch.int32)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda:0")
    bad[3] = bad[66] = True
    codes, scales = B.moe_mx4_quantize_rows(x)
    for y in (B.moe_grouped_gemm_mx4(codes, scales, off, *w1, activation=act), B.moe_grouped_ffn_mx4(x, off, *w1, *w2, activation=act)):
        assert torch.equal(torch.isnan(y), bad[:, None].expand_as(y))


def test_weights_past_four_gigabytes():
    K, N, E = 4096, 16384, 132                                                      # 4.4 GB of codes; the last expert's are behind 2^32 bytes
    rng = np.random.default_rng(13)
    print("mx4 product, weights of 4.4 GB", flush=True)
    codes = torch.zeros((E, N, K // 2), dtype=torch.uint8, device="cuda:0")
    scales = torch.full((E, K // 128, N, 4), 127, dtype=torch.uint8, device="cuda:0")
    c, s, values = held(rng, N, K, 0.02)
    codes[-1], scales[-1] = to_dev(c, torch.uint8), to_dev(s, torch.uint8)
    off = np.zeros(E + 1, dtype=np.int32)
    off[-1] = 5
    a = held(rng, 5, K)
    y = B.moe_grouped_gemm_mx4(*[to_dev(t, torch.uint8) for t in a[:2]], to_dev(off, torch.int32), codes, scales, y_dtype=torch.float32)
    check_rows(host(y.double()), a[2] @ values.T, np.abs(a[2]) @ np.abs(values).T, K, "f32", None)


def ffn_with_bounds(x, off, src, w1, w2, b1, b2, act):
    """y in 64 bits and how far another order of fc1's sums may move it: where h, moved by what fc1's error can be, takes another code or its block another
    scale, by the difference of the values times the weights."""
    _, _, xq = mx4.quantize(x)
    h, size = mx4.product(xq[src], off, w1, b1)
    n = off[-1]
    h, size, K = mx4.ACTIVATIONS[act](h[:n]), size[:n], x.shape[1]
    delta = 1.13 * (K / 64 + 9) * 2.0 ** -23 * size + (4e-7 * (np.abs(h) + size) if act == "gelu" else 0)
    _, _, hq = mx4.quantize(h)
    mag = np.abs(h).reshape(n, -1, 32)
    d = delta.reshape(n, -1, 32)
    lo, hi = (mag - d).clip(0).max(axis=2), (mag + d).max(axis=2)
    e_lo, e_hi = (mx4.exponents(np.repeat(t, 32, axis=1).reshape(n, -1)) for t in (lo, hi))
    v = [mx4.quantize(t, e)[2] for t in (h - delta, h + delta, h) for e in (e_lo, e_hi)]
    spread = np.max([np.abs(t - hq) for t in v], axis=0)
    y, size2 = mx4.product(hq, off, w2, b2)
    moved = np.zeros_like(y)
    for e in range(len(off) - 1):
        r = slice(off[e], off[e + 1])
        moved[r] = spread[r] @ np.abs(w2[e]).T
    return y, size2 + moved, moved, hq


FFN = [("few", 64, 64, "f16", False, "relu"), ("edges", 192, 320, "bf16", True, "relu"), ("tiles", 704, 576, "f16", True, "gelu"), ("tall", 256, 1024, "f32", False, "relu"),
       ("lone", 128, 192, "bf16", True, "gelu"), ("one", 1024, 4096, "f16", False, "relu"), ("many", 512, 256, "f16", True, "relu"), ("large", 192, 5568, "bf16", True, "relu")]


@pytest.mark.parametrize("load,d,F,dtype,bias,act", FFN)
def test_ffn(load, d, F, dtype, bias, act):
    print(f"mx4 ffn {load} d={d} F={F} {dtype} bias={bias} {act}", flush=True)
    rng = np.random.default_rng(d + F)
    rows, k = FFN_LOADS[load], 2
    E = len(rows)
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    R = int(off[-1]) + 1                                                            # the last row belongs to a pruned token
    R += R % k
    T = R // k
    src = rng.permutation(R).astype(np.int32)
    x = rows_of(rng, T, d, dtype)
    w1, w2 = experts_of(rng, E, d, F), experts_of(rng, E, F, d)
    b1, b2 = [(rng.standard_normal((E, n)) * 0.1).astype(np.float16) if bias else None for n in (F, d)]
    f = lambda t, dt: None if t is None else to_dev(t, dt)  # noqa: E731
    need = B.moe_grouped_ffn_mx4_workspace_bytes(T, R, d, F)
    results = []
    for fill in (0, 255):                                                           # whatever the workspace held before
        y = torch.full((R, d), -77.0, dtype=DT[dtype], device="cuda:0")
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda:0")
        B.moe_grouped_ffn_mx4(x, f(off, torch.int32), f(w1[0], torch.uint8), f(w1[1], torch.uint8), f(w2[0], torch.uint8), f(w2[1], torch.uint8),
                              b1=f(b1, torch.float16), b2=f(b2, torch.float16), perm_src=f(src, torch.int32), k=k, y_perm=y, activation=act, workspace=ws)
        results.append(y)
    assert torch.equal(*results)
    got, n = host(results[0].double()), off[-1]
    assert (got[n:] == -77.0).all()
    wide = lambda t: None if t is None else t.astype(np.float64)  # noqa: E731
    y, size, moved, _ = ffn_with_bounds(host(x.double()), off, src // k, w1[2], w2[2], wide(b1), wide(b2), act)
    tol = 1.13 * (F / 64 + 9) * 2.0 ** -23 * size[:n] + moved[:n]
    assert (np.abs(got[:n] - y[:n]) <= tol + ROUND[dtype] * (np.abs(y[:n]) + tol) + TINY[dtype]).all()
    print(f"   {(moved[:n] > 0).any(axis=1).mean():.3f} of the rows have an h on an edge", flush=True)


def test_h_is_quantised_as_rows_are():
    """With W2 = identity the FFN returns h's own 4-bit values: the epilogue's against the definition's, an expert with bias NaN included."""
    rng = np.random.default_rng(17)
    d, rows = 128, [33, 5, 2]
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    x = rng.standard_normal((40, d)).astype(np.float16)
    w1 = experts_of(rng, 3, d, d)
    eye = mx4.quantize(np.eye(d))
    b1 = (rng.standard_normal((3, d)) * 0.3).astype(np.float16)
    b1[1] *= np.float16(2.0 ** -9)
    b1[2, 70] = np.nan
    y = B.moe_grouped_ffn_mx4(to_dev(x, torch.float16), to_dev(off, torch.int32), to_dev(w1[0], torch.uint8), to_dev(w1[1], torch.uint8),
                              to_dev(np.stack([eye[0]] * 3), torch.uint8), to_dev(np.stack([eye[1]] * 3), torch.uint8), b1=to_dev(b1, torch.float16), y_dtype=torch.float32,
                              activation="gelu")
    got = host(y).astype(np.float64)
    want, _, moved, hq = ffn_with_bounds(x.astype(np.float64), off, np.arange(40), w1[2], np.stack([eye[2]] * 3), b1.astype(np.float64), None, "gelu")
    assert np.isnan(got[38:]).all()                 # (a block that is not a number spoils every sum it takes part in)
    assert (np.abs(got[:38] - hq[:38]) <= moved[:38]).all()


def test_empty_calls_and_a_graph():
    E, d, F = 3, 128, 256
    rng = np.random.default_rng(19)
    w1, w2 = [[to_dev(t, torch.uint8) for t in experts_of(rng, E, a, b)[:2]] for a, b in ((d, F), (F, d))]
    off = torch.zeros(E + 1, dtype=torch.int32, device="cuda:0")
    assert B.moe_grouped_ffn_mx4(torch.empty((0, d), dtype=torch.float16, device="cuda:0"), off, *w1, *w2).shape == (0, d)
    codes, scales = B.moe_mx4_quantize_rows(torch.empty((0, d), dtype=torch.float16, device="cuda:0"))
    assert codes.shape == (0, d // 2) and B.moe_mx4_dequantize(codes, scales).shape == (0, d)
    x = torch.empty((24, d), dtype=torch.float16, device="cuda:0")
    y, ws = torch.empty_like(x), torch.empty(B.moe_grouped_ffn_mx4_workspace_bytes(24, 24, d, F), dtype=torch.uint8, device="cuda:0")
    call = lambda: B.moe_grouped_ffn_mx4(x, off, *w1, *w2, y_perm=y, workspace=ws)  # noqa: E731
    inputs = [(to_dev(rng.standard_normal((24, d)), torch.float16), to_dev(np.array(o), torch.int32)) for o in ([0, 1, 9, 24], [0, 24, 24, 24], [0, 0, 0, 20])]
    eager = []
    for xi, oi in inputs:
        x.copy_(xi), off.copy_(oi), y.zero_()
        eager.append(call().clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(2):
        for (xi, oi), want in zip(inputs, eager):
            x.copy_(xi), off.copy_(oi), y.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
