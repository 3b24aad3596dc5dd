"""AdamW over many tensors against the formula in 64 bits; states in 8 bits against their definition, value by value."""
import math

import pytest
import torch

from paper_2211_10017_amd import binding as B
from tuning_ref import BF16, F16, F32, U, generator, half_step

pytestmark = pytest.mark.gpu
ARGS = dict(lr=1e-2, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1, grad_scale=0.5)


def held(codes, scales):
    """The values of a state in 8 bits, in 64."""
    s = scales.double() - 127
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(s).repeat_interleave(32)[:codes.numel()]


def quantised(v, root):
    """Codes' values, and the scales, that v (64 bits, of fp32 numbers) has by the definition."""
    n = v.numel()
    b = torch.nn.functional.pad(v, (0, -n % 32)).view(-1, 32)
    top = b.abs().amax(1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 8, -127).clamp(min=-127)
    a = b.abs() * torch.exp2(-e.double())
    step = torch.exp2((torch.frexp(a)[1] - 4).clamp(min=-9).double())
    q = torch.round(a / step) * step
    if root:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    fine = torch.isfinite(top)                            # a block with an infinity is not a number
    value = torch.where(fine, torch.sign(b) * q * torch.exp2(e.double()), math.nan)
    return value.view(-1)[:n], torch.where(fine, e + 127, 255).view(-1), (step * torch.exp2(e.double())).view(-1)[:n]


def want_step(p, g, m, v, t, lr, betas, eps, weight_decay, grad_scale):
    """p, m, v after a step in 64 bits, and how far fp32 arithmetic may be off."""
    b1, b2 = betas
    g = g.double() * grad_scale
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    dm, dv = 4 * U * (b1 * m.abs() + (1 - b1) * g.abs()), 6 * U * v1                 # products, factors and the sum: at most four (six) roundings of the terms
    rate, root = lr / (1 - b1 ** t), 1 / math.sqrt(1 - b2 ** t)
    den = torch.sqrt(v1) * root + eps
    move = rate * m1 / den
    dp = rate * dm / den + 12 * U * move.abs() + 4 * U * p.double().abs()             # v's 6 roundings halve under the root; root, product, sum, quotient, rate
    return p.double() * (1 - lr * weight_decay) - move, m1, v1, dp, dm, dv


def tensors(gen, sizes, pd, gd, offset=0):
    """A list of tensors each `offset` values behind a 16-byte border."""
    def make(n, dtype, f):
        room = torch.empty(n + offset, dtype=dtype, device="cuda")
        t = room[offset:]
        return t.copy_(f(n))
    r = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    p = [make(n, pd, lambda n: r(n) * 0.1) for n in sizes]
    g = [make(n, gd, lambda n: r(n) * torch.exp(r(n))) for n in sizes]
    m = [make(n, F32, lambda n: r(n) * 0.1) for n in sizes]
    v = [make(n, F32, lambda n: r(n).square() * 0.1 + 1e-6) for n in sizes]
    return p, g, m, v


@pytest.mark.parametrize("pd,gd,copy", [(F32, F32, None), (F32, BF16, BF16), (F32, F16, F16), (F16, F16, None), (BF16, BF16, None), (BF16, F32, None), (F32, F32, F16), (F16, F32, None)])
@pytest.mark.parametrize("sizes", [[1], [31, 32, 33], [4096, 4097, 5, 1, 0, 70001], [3] * 100])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_32_bits(pd, gd, copy, sizes, offset):
    print(f"adamw 32 {pd} {gd} {copy} {sizes[:6]} +{offset}", flush=True)
    gen = generator(len(sizes))
    p, g, m, v = tensors(gen, sizes, pd, gd, offset)
    copies = [torch.empty(n + offset, dtype=copy, device="cuda")[offset:] for n in sizes] if copy else None
    for t in (1, 2, 1000):
        wants = [want_step(*x, t, **ARGS) for x in zip(p, g, [x.double() for x in m], [x.double() for x in v])]
        B.moe_adamw(p, g, m, v, t, copies=copies, **ARGS)
        torch.cuda.synchronize()
        for i, (wp, wm, wv, dp, dm, dv) in enumerate(wants):
            assert bool(((p[i].double() - wp).abs() <= dp + half_step(wp.abs() + dp, pd)).all()), (t, i)
            assert bool(((m[i].double() - wm).abs() <= dm).all()) and bool(((v[i].double() - wv).abs() <= dv).all()), (t, i)
            if copy:
                assert torch.equal(copies[i], p[i].to(copy))


@pytest.mark.parametrize("pd,gd,copy", [(F32, F32, None), (F32, BF16, BF16), (BF16, BF16, None), (F16, F32, None)])
@pytest.mark.parametrize("sizes", [[1], [31, 32, 33], [4096, 4097, 5, 1, 0, 70001], [3] * 100])
@pytest.mark.parametrize("offset", [0, 1])
def test_states_in_8_bits(pd, gd, copy, sizes, offset):
    """p as from the values that the states stand for; the states the codes of the new ones, of the neighbouring number at most where fp32 rounding meets a border."""
    print(f"adamw 8 {pd} {gd} {copy} {sizes[:6]} +{offset}", flush=True)
    gen = generator(len(sizes))
    p, g, _, _ = tensors(gen, sizes, pd, gd, offset)
    zeros = lambda n: torch.zeros(n + offset, dtype=torch.uint8, device="cuda")[offset:]  # noqa: E731
    m, v = ([(zeros(n), zeros((n + 31) // 32)) for n in sizes] for _ in range(2))
    copies = [torch.empty(n + offset, dtype=copy, device="cuda")[offset:] for n in sizes] if copy else None
    for t in (1, 2, 3):
        old = [(held(*x), held(*y)) for x, y in zip(m, v)]
        wants = [want_step(q, h, x, r * r, t, **ARGS) for q, h, (x, r) in zip(p, g, old)]
        B.moe_adamw(p, g, m, v, t, copies=copies, **ARGS)
        torch.cuda.synchronize()
        for i, (wp, wm, wv, dp, dm, dv) in enumerate(wants):
            if not sizes[i]:
                continue
            assert bool(((p[i].double() - wp).abs() <= dp + half_step(wp.abs() + dp, pd)).all()), (t, i)
            if copy:
                assert torch.equal(copies[i], p[i].to(copy))
            for state, new, slack, root in ((m[i], wm, dm, False), (v[i], wv.sqrt(), 4 * U * wv.sqrt(), True)):
                value, scale, step = quantised(new, root)
                got = held(*state)
                # (numbers near 0 are whole multiples of 2^-9 units of the scale that the block has, which may be the next one, see below)
                step = torch.maximum(step, torch.exp2(state[1].double() - 136).repeat_interleave(32)[:sizes[i]])
                assert bool(((got - new).abs() <= step / 2 + slack + torch.where((got - value) == 0, step, 0.0)).all()), (t, i, root)      # (the smallest root is rounded up)
                # Codes and scales that differ are not counted: the first step's root is |g| / 20, which lies halfway between two codes wherever the mantissa of g, eight bits in
                # bf16, is five times an odd number of five (one g in sixteen), and on a power of two where it is five; there fp32's rounding of the factors decides.  A scale may
                # differ only there: the largest of the 32 is then within its slack of a power of two.
                top, most = (torch.nn.functional.pad(t, (0, -sizes[i] % 32)).view(-1, 32).amax(1) for t in (new.abs(), slack))
                border = torch.exp2(torch.round(torch.log2(top.clamp(min=1e-300))))
                assert bool(((state[1].double() == scale) | ((top - border).abs() <= most)).all()), (t, i, root)
                back = B.moe_adamw_state(*state, F32)
                assert torch.equal(back.double(), got) and torch.equal(B.moe_adamw_state(*state, BF16).double(), got)


def test_8_bit_codes_are_the_definitions():
    """A step that leaves a chosen m behind (beta1 = 0: m = g), of every kind of value: borders between codes, subnormal numbers, blocks of zeros, one large value, infinities and NaN."""
    gen = generator(5)
    grid = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()
    grid = grid[grid <= 256]
    borders = (grid[1:] + grid[:-1]) / 2
    near = torch.cat([grid, borders, borders * (1 + 2.0 ** -20), borders * (1 - 2.0 ** -20)])
    rows = []
    for unit in (2.0 ** -126, 2.0 ** -100, 1.0, 2.0 ** 100):
        for part in near.split(30):
            rows.append(torch.nn.functional.pad(torch.cat([torch.tensor([255.0, 128.5], device="cuda"), part]), (0, 30 - len(part))) * unit)
    rows += [torch.zeros(32, device="cuda"), torch.full((32,), 2.0 ** -140, device="cuda"), torch.randn(32, generator=gen, device="cuda") * 1e-42]
    m = torch.cat(rows) * torch.where(torch.rand(32 * len(rows), generator=gen, device="cuda") < 0.5, -1.0, 1.0)
    n = m.numel()
    codes = lambda: (torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n // 32, dtype=torch.uint8, device="cuda"))  # noqa: E731
    sm, sv = codes(), codes()
    B.moe_adamw([torch.zeros(n, device="cuda")], [m], [sm], [sv], 1, betas=(0.0, 0.5))
    value, scale, _ = quantised(m.double(), False)
    assert torch.equal(held(*sm), value) and torch.equal(sm[1].long(), scale.long())
    value, scale, _ = quantised(torch.sqrt(m * m * 0.5).double(), True)                     # (the largest squares are infinities in fp32)
    assert torch.equal(sv[1].long(), scale.long())
    assert torch.equal(torch.where((sv[1] == 255).repeat_interleave(32), 0.0, held(*sv)), value.nan_to_num(0.0)) and bool(torch.isnan(B.moe_adamw_state(*sv)[torch.isnan(value)]).all())
    for bad in (float("inf"), float("nan"), -float("inf")):
        g = m.clone()
        g[40] = bad
        sm, sv = codes(), codes()
        B.moe_adamw([torch.zeros(n, device="cuda")], [g], [sm], [sv], 1, betas=(0.0, 0.5))
        assert int(sm[1][1]) == 255 and int(sv[1][1]) == 255 and bool(torch.isnan(B.moe_adamw_state(*sm)[32:64]).all())
        want = quantised(m.double(), False)[0]
        assert torch.equal(held(*sm)[64:], want[64:]) and torch.equal(held(*sm)[:32], want[:32])


def test_a_small_root_beside_a_large_one_stays_above_zero():
    """A step whose gradient has gone to 0 for a value with a small second moment: m / sqrt(v) stays within what 8 bits can say, far from m / eps."""
    n = 32
    p, sm, sv = torch.zeros(n, device="cuda"), *(tuple(torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, 1)) for _ in range(2))
    g = torch.full((n,), 1e-6, device="cuda")
    g[0] = 1e6
    B.moe_adamw([p], [g], [sm], [sv], 1, lr=0.0, weight_decay=0.0)
    assert bool((held(*sv) > 0).all())
    B.moe_adamw([p], [torch.zeros_like(g)], [sm], [sv], 2, lr=1.0, weight_decay=0.0)
    assert float(p.abs().max()) < 4


@pytest.mark.parametrize("bits", [32, 8])
def test_the_step_number_on_the_device(bits):
    """Captured and replayed with a counter that the graph advances: the same bits as steps numbered by the host, several replays."""
    gen = generator(bits)
    sizes = [1000, 33, 4096]

    def fresh():
        g2 = generator(8)
        p, g, m, v = tensors(g2, sizes, F32, BF16)
        if bits == 8:
            m, v = ([(torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda")) for n in sizes] for _ in range(2))
        return p, g, m, v

    flat = lambda s: [x for t in s for x in (t if isinstance(t, tuple) else (t,))]  # noqa: E731
    a, b = fresh(), fresh()
    step = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        B.moe_adamw(*a, step, **ARGS)
    for t in range(1, 6):
        for x, y in zip(a[1], b[1]):
            x.normal_(generator=gen)
            y.copy_(x)
        graph.replay()
        B.moe_adamw(*b, t, **ARGS)
        torch.cuda.synchronize()
        for x, y in zip(flat(a[0]) + flat(a[2]) + flat(a[3]), flat(b[0]) + flat(b[2]) + flat(b[3])):
            assert torch.equal(x, y), t


def test_a_large_tensor_reaches_past_32_bits():
    n = (1 << 31) + 12345
    p = torch.zeros(n, dtype=BF16, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    g[-5:] = 1.0
    g[7] = -1.0
    state = lambda: (torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda"))  # noqa: E731
    m, v = state(), state()
    B.moe_adamw([p], [g], [m], [v], 1, lr=0.5, weight_decay=0.0)
    torch.cuda.synchronize()
    assert int((p != 0).sum()) == 6 and bool((p[-5:] == -0.5).all()) and float(p[7]) == 0.5
    assert int((m[0] != 0).sum()) == 6 and float(B.moe_adamw_state(*m, BF16)[-1]) > 0
