"""The largest counts that the 4-bit operators and the balance loss take, on the host, before anything is launched."""
import ctypes

import pytest

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
