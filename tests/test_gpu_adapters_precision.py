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


def coefficient(dtype, result):
    """How far a coefficient's 16-bit terms are off, relative to it: two terms of 8 bits (half a step 2^-8 each) or, where the result is fp32, three of bf16; two of 11 bits in fp16; fp32 rows meet
    fp32 coefficients."""
    return 0.0 if dtype == F32 else 2.0 ** -22 if dtype == F16 else 2.0 ** -24 if result == F32 else 2.0 ** -16


def check(x, a, b, offsets, perm, k, scale, by, y, dy, out_dt, grad_dt):
    """Forward and backward against the formulas in 64 bits.  Bounds: a sum of n products is off by n roundings of the sum of their magnitudes (three terms of a coefficient are three products), a
    coefficient by that of its own sum and by its terms, fp16 ones at least by 2^-25 units, a unit being 2^-14 of the largest (of a row; of the rows and ranks for the matrices) or less."""
    want = adapters_ref(x, a, b, offsets, perm, k, scale, by, y, dy)
    E, rank, K = a.shape
    N, R, dt = b.shape[2], dy.shape[0], x.dtype
    v = torch.empty((R, rank), device="cuda")
    out = B.moe_adapters(x, a, b, offsets, perm, k, scale, by, y=y, y_dtype=out_dt, v=v)
    dx, da, db = B.moe_adapters_backward(dy, x, a, b, v, offsets, perm, k, scale, by, grad_dtype=grad_dt)
    torch.cuda.synchronize()
    source, off = perm.long(), offsets.tolist()
    place = source if by else torch.arange(R, device="cuda")

    def near(name, got, target, sums, terms, extra=0.0):
        w = target.double()
        slack = sums + terms + extra + (2.0 ** -25 if got.dtype == F16 else 0.0)
        miss = (got.double() - w).abs() - (slack + half_step(w.abs() + slack, got.dtype))
        assert bool((miss <= 0).all()), (name, float(miss.max()))

    floor = 2.0 ** -39 if dt == F16 else 0.0
    for e in range(E):
        rows = slice(off[e], off[e + 1])
        n = off[e + 1] - off[e]
        if n == 0:
            assert bool((da[e] == 0).all()) and bool((db[e] == 0).all())
            continue
        s = 1.0 if scale is None else float(scale[e])
        xe, ae, be, de = x[source[rows] // k].double(), a[e].double(), b[e].double(), dy[place[rows]].double()
        ve, vm = xe @ ae.T, xe.abs() @ ae.abs().T
        ue, um = s * (de @ be.T), s * (de.abs() @ be.abs().T)
        near("v", v[rows], ve, K * U * vm, 0.0)
        added = 0.0 if y is None else U * (y[place[rows]].double().abs() + want["out"][place[rows]].abs())
        near("out", out[place[rows]], want["out"][place[rows]], (K + 3 * rank + 2) * U * s * (vm @ be.abs()), coefficient(dt, out_dt) * s * (ve.abs() @ be.abs()),
             floor * s * ve.abs().amax(1, keepdim=True) * be.abs().sum(0) + added)
        near("dx", dx[place[rows]], want["dx"][place[rows]], (N + 3 * rank + 2) * U * (um @ ae.abs()), coefficient(dt, dt) * (ue.abs() @ ae.abs()), floor * ue.abs().amax(1, keepdim=True) * ae.abs().sum(0))
        near("da", da[e], want["da"][e], (N + 3 * n + 2) * U * (um.T @ xe.abs()), coefficient(dt, grad_dt) * (ue.abs().T @ xe.abs()), floor * ue.abs().max() * xe.abs().sum(0))
        near("db", db[e], want["db"][e], (K + 3 * n + 3) * U * s * (vm.T @ de.abs()), coefficient(dy.dtype, grad_dt) * s * (ve.abs().T @ de.abs()),
             (2.0 ** -39 if dy.dtype == F16 else 0.0) * s * ve.abs().max() * de.abs().sum(0))
    rest = place[off[E]:]
    assert bool((dx[rest] == 0).all()) and torch.equal(out[rest], torch.zeros_like(out[rest]) if y is None else y[rest])


TYPES = [(F16, F16), (F16, F32), (BF16, BF16), (BF16, F32), (F16, BF16), (BF16, F16)]


@pytest.mark.parametrize("dt,yt", TYPES)
@pytest.mark.parametrize("grad_dt", [F32, None])
@pytest.mark.parametrize("R,K,N,rank", [(3, 8, 8, 1), (6, 8, 16, 2), (40, 16, 8, 3), (6, 40, 8, 17), (5, 8, 24, 70)])
def test_terms_of_coefficients(R, K, N, rank, dt, yt, grad_dt):
    """Few channels and rows: what the sums themselves are off by is far below a lost term."""
    print(f"terms R={R} K={K} N={N} rank={rank} {dt} {yt} {grad_dt}", flush=True)
    gen, E = generator(R + rank), 2
    perm, _, offsets = sorted_index(routing(gen, R, 1, E, "even"), E)
    x, a, b, dy = r(gen, R, K).to(dt), r(gen, E, rank, K).to(dt), r(gen, E, rank, N).to(dt), r(gen, R, N).to(yt)
    check(x, a, b, offsets, perm, 1, torch.rand(E, generator=gen, device="cuda") + 0.5, False, None, dy, yt, grad_dt or dt)


# Blocks of up to 16, 32, 48 and 64 or 80 rows: a block's share is a 248th of all rows, or of a part of them where that is more than a block holds.
@pytest.mark.parametrize("dt,yt", TYPES)
@pytest.mark.parametrize("R,rank", [(4700, 16), (4700, 24), (9001, 9), (9001, 32), (14999, 16), (14999, 20), (14999, 32), (17800, 5), (24000, 32), (14000, 64), (9001, 64), (13500, 64), (14000, 100), (9900, 100)])
@pytest.mark.parametrize("load,k,by", [("even", 1, True), ("pruned", 2, False), ("ends", 2, False)])
def test_every_size_of_block(R, rank, dt, yt, load, k, by):
    print(f"blocks R={R} rank={rank} {dt} {yt} {load} k={k}", flush=True)
    gen, E, K, N = generator(R + rank), 7, 72, 136
    T = R // k
    perm, _, offsets = sorted_index(routing(gen, T, k, E, load), E)
    x, a, b = r(gen, T, K).to(dt), (r(gen, E, rank, K) * K ** -0.5).to(dt), r(gen, E, rank, N).to(dt)
    y, dy = r(gen, T * k, N).to(yt), r(gen, T * k, N).to(yt)
    check(x, a, b, offsets, perm, k, torch.rand(E, generator=gen, device="cuda") + 0.5, by, y if load != "ends" else None, dy, yt, F32 if load == "even" else dt)
