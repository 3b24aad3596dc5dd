"""The largest counts that the 4-bit operators and the balance loss take, on the host, before anything is launched."""
import ctypes

import pytest

from launches import P as PTR, record
from paper_2211_10017_amd import binding as B

P = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
ARG, UNSUPPORTED, WORKSPACE = 1, 2, 3
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    return B.load()


def test_assignments_are_counted_in_32_bits(lib):
    """counts is int32 and so is the sum of them."""
    fwd = lambda T, k, E=8, size=0: lib.moe_balance_loss(P, 1, P, T, E, k, 1, 0.01, P, P, P, P, P, P, size, None)  # noqa: E731
    back = lambda T, k, out=P, E=8: lib.moe_balance_loss_backward(P, 1, P, T, E, k, 1, P, None, None, out, None)  # noqa: E731
    for T, k in ((2 ** 28, 8), (2 ** 30, 2), (MOST, 2)):
        assert fwd(T, k) == ARG and b"T*k" in lib.moe_last_error()
        assert back(T, k) == ARG and b"T*k" in lib.moe_last_error()
    for T, k in ((2 ** 28 - 1, 8), (2 ** 30 - 1, 2), (MOST, 1)):
        assert fwd(T, k) == WORKSPACE                                              # (what a call is refused for that goes past the counts)
        assert back(T, k, None) == ARG and b"NULL" in lib.moe_last_error()


def test_rows_that_a_lanes_offsets_reach(lib):
    """A lane finds its row's scales by four bytes times the row's number in 32 bits: fewer than 2^30 rows, those of h as well, which are R."""
    ffn = lambda T, R: lib.moe_grouped_ffn_mx4(P, 0, T, P, 1, P, R, 2, 0, 64, 64, 0, P, P, None, P, P, None, P, 0, P, 0, None)  # noqa: E731
    gemm = lambda rows, R, y=P: lib.moe_grouped_gemm_mx4(P, P, rows, P, 1, P, R, 2, 0, 64, 32, P, P, None, -1, y, 0, None)  # noqa: E731
    assert ffn(2 ** 30, 8) == UNSUPPORTED and ffn(8, 2 ** 30) == UNSUPPORTED and b"2^30" in lib.moe_last_error() and ffn(8, MOST) == UNSUPPORTED
    assert ffn(2 ** 30 - 1, 2 ** 30 - 1) == WORKSPACE
    assert gemm(2 ** 30, 8) == UNSUPPORTED and gemm(8, MOST, None) == ARG          # (a product's R is only how many rows it writes)


def test_more_rows_than_a_launch_takes(lib):
    for R in (2 ** 28 + 16, MOST - 15, MOST - 14, MOST):
        for dtype in (0, 1, 2):
            assert lib.moe_mx4_quantize_rows(P, dtype, R, 64, 64, P, P, None) == UNSUPPORTED and b"exceed one launch" in lib.moe_last_error()
            assert lib.moe_mx4_dequantize(P, P, 1, R, 64, P, dtype, None) == UNSUPPORTED and b"exceed one launch" in lib.moe_last_error()
    assert lib.moe_mx4_quantize_rows(P, 0, 40000, MOST - 63, MOST - 63, P, P, None) == UNSUPPORTED
    assert lib.moe_mx4_quantize_experts(P, 1, MOST - 63, 64, P, P, None) == UNSUPPORTED
    assert lib.moe_mx4_quantize_experts(P, 1, 64, MOST - 31, P, P, None) == UNSUPPORTED and lib.moe_mx4_dequantize(P, P, 1, 64, MOST - 63, P, 0, None) == UNSUPPORTED


def test_the_longest_row_takes_a_launch():
    one = record([("moe_mx4_quantize_rows", [PTR, 0, 1, MOST - 63, [MOST - 63], PTR, PTR, None])])[0]
    assert one.rc == 0 and one.launches[0].grid[0] == 2 ** 24 // 4
