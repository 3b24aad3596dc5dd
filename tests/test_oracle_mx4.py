"""What fixes the oracle of the 4-bit format and of the balance loss other than itself: printed values, hand-worked blocks, brute force, differences."""
import numpy as np
import pytest

from oracle import mx4


def test_the_numbers_of_the_format():
    codes = np.arange(16, dtype=np.uint8)
    row = np.zeros((1, 16), dtype=np.uint8)
    row[0, :8] = codes[0::2] | (codes[1::2] << 4)
    got = mx4.dequantize(np.tile(row, (1, 2)), np.array([[[127, 130, 0, 0]]], dtype=np.uint8))[0]
    want = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6])
    assert (got[:16] == want).all() and (got[32:48] == 8 * want).all() and not got[16:32].any()


def test_a_block_worked_by_hand():
    v = np.zeros((1, 64))
    v[0, :14] = [7.9, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -5.001, -0.2501, 6.0, -0.0, 0.24, 4.999]      # largest below 8: unit 1
    v[0, 32:36] = [8.0, 1.0, -1.5, 3.0]                                                                        # 8: unit 2
    codes, scales, values = mx4.quantize(v)
    assert scales[0, 0].tolist() == [127, 128, 0, 0]
    assert values[0, :14].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -6, -0.5, 6, 0, 0, 4]
    assert values[0, 32:36].tolist() == [8, 1, -2, 3]                   # -0.75 of the unit is halfway: to the even code, 1
    assert (mx4.dequantize(codes, scales) == values).all()


def test_nearest_by_brute_force_and_scales_at_their_ends():
    a = np.concatenate([np.linspace(0, 8, 4097), (mx4.GRID[1:] + mx4.GRID[:-1]) / 2])
    for x, i in zip(a, mx4.nearest_code(a)):
        d = np.abs(mx4.GRID - x)
        best = np.flatnonzero(d == d.min())
        assert i in best and (len(best) == 1 or i % 2 == 0)
    v = np.zeros((1, 32 * 8))
    v[0, 0::32] = [np.float32(2.0 ** -149), 2.0 ** -126, 2.0 ** -125, 2.0 ** -124, float(np.finfo(np.float32).max), np.inf, np.nan, 0.0]
    assert mx4.exponents(v)[0].tolist() == [-127, -127, -127, -126, 125, 128, 128, -127]
    assert np.isnan(mx4.quantize(v)[2][0, 5 * 32:7 * 32]).all()


@pytest.mark.parametrize("k,renorm", [(1, False), (1, True), (2, False), (2, True), (3, True)])
def test_balance_gradient_against_differences(k, renorm):
    rng = np.random.default_rng(k)
    T, E = 7, 5
    z = rng.standard_normal((T, E))
    idx = np.argsort(-z, axis=1)[:, :k].astype(np.int32)
    idx[2] = E
    if k > 1:
        idx[3, 1] = E                                                       # one slot of a token without an expert
    ds = rng.standard_normal((T, k))
    f = lambda z: (lambda r: 0.7 * r["loss"] + (ds * r["scale"])[idx < E].sum())(mx4.balance(z, idx, 0.3, renorm))  # noqa: E731
    grad = mx4.balance(z, idx, 0.3, renorm, 0.7, ds)["dlogits"]
    for t in range(T):
        for e in range(E):
            d = np.zeros_like(z)
            d[t, e] = 1e-5
            assert abs((f(z + d) - f(z - d)) / 2e-5 - grad[t, e]) < 1e-8


def test_balance_loss_is_one_coefficient_at_balance_and_all_of_them_at_collapse():
    T, E = 64, 8
    even = mx4.balance(np.zeros((T, E)), (np.arange(T)[:, None] % E).astype(np.int32), 0.01, False)
    assert abs(even["loss"] - 0.01) < 1e-15 and (even["counts"] == T // E).all()
    z = np.full((T, E), -50.0)
    z[:, 3] = 50
    assert abs(mx4.balance(z, np.full((T, 1), 3, dtype=np.int32), 0.01, False)["loss"] - 0.08) < 1e-12
