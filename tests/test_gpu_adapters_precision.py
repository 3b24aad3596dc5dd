"""How precise the adapters' products are, type by type, where few summands let the coefficients' own rounding be seen; coefficients that are not finite; and every size of block."""
import pytest
import torch

from paper_2211_10017_amd import binding as B
from tuning_ref import BF16, F16, F32, U, adapters_ref, generator, half_step, routing, sorted_index

pytestmark = pytest.mark.gpu


def r(gen, *s):
    return torch.randn(s, generator=gen, device="cuda")


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rank", [3, 20, 40])
@pytest.mark.parametrize("rows", [5, 90])
def test_a_coefficient_that_is_not_finite_is_its_ranks_alone(rows, rank, dtype, bad):
    """db[j] = sum_r v[r][j] dy[r]: one v that is no number, and the other ranks' sums are as without it."""
    gen, E, C = generator(rows + rank), 2, 72
    offsets = torch.tensor([0, rows, rows], dtype=torch.int32, device="cuda")
    dy, a, b = r(gen, rows, C).to(dtype), r(gen, E, rank, 64).to(dtype), r(gen, E, rank, C).to(dtype)
    v = r(gen, rows, rank)
    plain = B.moe_adapters_backward(dy, None, a, b, v, offsets, need=(False, False, True), grad_dtype=F32)[2]
    for row in {0, rows // 2, rows - 1}:
        one = v.clone()
        one[row, 1] = bad
        got = B.moe_adapters_backward(dy, None, a, b, one, offsets, need=(False, False, True), grad_dtype=F32)[2]
        others = [j for j in range(rank) if j != 1]
        want, most = v[:, others].double().T @ dy.double(), v[:, others].double().abs().T @ dy.double().abs()
        # sums of `rows` products; coefficients in two fp16 terms are off by 2^-22, in three of bf16 by 2^-24
        assert bool(((got[0][others].double() - want).abs() <= ((rows + 4) * U + 2.0 ** -22) * most).all())
        assert not bool(torch.isfinite(got[0][1]).any()) and bool((got[1] == 0).all())
        if dtype == BF16:
            assert torch.equal(got[0][others], plain[0][others])


@pytest.mark.parametrize("value,want", [(3.395e38, 3.395e38), (3.4e38, float("inf"))])
def test_coefficients_about_the_largest_bf16_number(value, want):
    """The largest bf16 number is (2 - 2^-7) 2^127 = 3.3895e38; up to half a step above it, (2 - 2^-8) 2^127 = 3.3962e38, numbers are rounded to it and the other terms hold the rest.  Above that, where
    only fp32 is finite, they count as infinite (what is left of them, minus an infinity, would make a NaN of every sum)."""
    offsets = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    a, b, dy = (torch.ones(s, dtype=BF16, device="cuda") for s in ((1, 2, 64), (1, 2, 64), (1, 64)))
    v = torch.tensor([[value, 1.0]], device="cuda")
    want = torch.tensor(want, device="cuda")
    near = lambda t: bool((t == want).all() if torch.isinf(want) else ((t - want).abs() <= 2.0 ** -22 * want).all())  # noqa: E731
    db = B.moe_adapters_backward(dy, None, a, b, v, offsets, need=(False, False, True), grad_dtype=F32)[2]
    assert near(db[0, 0]) and bool((db[0, 1] == 1).all())
    x = torch.zeros((1, 64), dtype=BF16, device="cuda")
    x[0, 0] = 1.0
    a[0, 1] = 0.0
    assert near(B.moe_adapters(x, a, b, offsets, scale=torch.tensor([value], device="cuda"), y_dtype=F32))
