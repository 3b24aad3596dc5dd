"""Gradient of sorting tokens by expert and back: moe_combine_backward and moe_permute_backward against the formulas in 64 bits, with pruned rows that hold
anything, and through autograd-like differences of the forward calls."""
import pytest
import torch

from paper_2211_10017_amd import binding as B
from tuning_ref import BF16, F16, F32, U, generator, routing, sorted_index, within

pytestmark = pytest.mark.gpu
SIZES = [(1, 1, 8), (1, 2, 8), (33, 1, 64), (257, 2, 72), (5, 3, 128), (129, 2, 1032), (64, 8, 520), (1000, 2, 704)]


@pytest.mark.parametrize("out_dt,y_dt", [(F32, F16), (F32, F32), (F16, F16), (BF16, BF16), (BF16, F32), (F16, BF16), (F32, BF16), (BF16, F16), (F16, F32)])
@pytest.mark.parametrize("T,k,d", SIZES)
@pytest.mark.parametrize("load", ["even", "pruned"])
def test_combine_backward(T, k, d, out_dt, y_dt, load):
    print(f"combine_backward T={T} k={k} d={d} {out_dt} {y_dt} {load}", flush=True)
    gen, E = generator(T + k + d), 8
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, load), E)
    R, active = T * k, int(offsets[E])
    dout = torch.randn((T, d), generator=gen, device="cuda").to(out_dt)
    y = torch.randn((R, d), generator=gen, device="cuda").to(y_dt)
    y[active:] = float("nan")
    scale = torch.rand((T, k), generator=gen, device="cuda")
    dy, dscale = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:])
    again = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:])
    torch.cuda.synchronize()
    live = inv.long() < active
    o = dout.double().repeat_interleave(k, 0)
    rows = torch.where(live[:, None], y.double()[inv.long()], 0.0)
    want = torch.zeros((R, d), dtype=torch.float64, device="cuda")
    want[inv.long()] = torch.where(live[:, None], scale.double().view(-1, 1) * o, 0.0)
    within(dy, want, U * want.abs())
    within(dscale, (o * rows).sum(1).view(T, k), (d + 1) * U * (o * rows).abs().sum(1).view(T, k))
    assert bool((dy[active:] == 0).all()) and bool((dscale[~live.view(T, k)] == 0).all())
    assert torch.equal(again[0], dy) and torch.equal(again[1], dscale)
    only = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:], need=(True, False))
    assert torch.equal(only[0], dy) and only[1] is None
    only = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:], need=(False, True))
    assert only[0] is None and torch.equal(only[1], dscale)


@pytest.mark.parametrize("in_dt,out_dt", [(F16, F16), (BF16, BF16), (F32, F32), (F32, BF16), (F16, F32), (BF16, F32), (F32, F16), (F16, BF16), (BF16, F16)])
@pytest.mark.parametrize("T,k,d", SIZES)
@pytest.mark.parametrize("load", ["even", "pruned"])
def test_permute_backward(T, k, d, in_dt, out_dt, load):
    print(f"permute_backward T={T} k={k} d={d} {in_dt} {out_dt} {load}", flush=True)
    gen, E = generator(T + k + d), 8
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, load), E)
    active = int(offsets[E])
    g = torch.randn((T * k, d), generator=gen, device="cuda").to(in_dt)
    g[active:] = float("nan")
    dx = B.moe_permute_backward(g, inv, T, k, active_rows=offsets[E:], out_dtype=out_dt)
    torch.cuda.synchronize()
    rows = torch.where((inv.long() < active)[:, None], g.double()[inv.long()], 0.0).view(T, k, d)
    within(dx, rows.sum(1), k * U * rows.abs().sum(1))


def test_no_tokens():
    for k in (1, 2):
        empty = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
        index = torch.empty(0, dtype=torch.int32, device="cuda")
        dy, ds = B.moe_combine_backward(empty(0, 64), empty(0, 64), index, empty(0, k))
        assert dy.shape == (0, 64) and ds.shape == (0, k) and B.moe_permute_backward(empty(0, 64), index, 0, k).shape == (0, 64)


def test_every_row_pruned_and_no_count():
    gen = generator(3)
    T, k, d, E = 40, 2, 64, 4
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, "none"), E)
    y, dout, scale = torch.full((T * k, d), float("inf"), device="cuda"), torch.ones((T, d), device="cuda"), torch.ones((T, k), device="cuda")
    dy, ds = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:])
    assert bool((dy == 0).all()) and bool((ds == 0).all()) and bool((B.moe_permute_backward(y, inv, T, k, active_rows=offsets[E:]) == 0).all())
    # without active_rows every row counts
    dy, ds = B.moe_combine_backward(dout, torch.ones_like(y), inv, scale)
    assert bool((dy == 1).all()) and bool((ds == d).all()) and bool((B.moe_permute_backward(dy, inv, T, k) == k).all())


@pytest.mark.parametrize("k", [1, 2])
def test_some_tokens_of_a_batch(k):
    """A call for some of the tokens writes their rows of the batch's dy and no others; indices outside the rows are read as pruned."""
    gen = generator(k)
    T, d, E = 100, 72, 8
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, "pruned"), E)
    y, dout = torch.randn((T * k, d), generator=gen, device="cuda"), torch.randn((T, d), generator=gen, device="cuda")
    scale = torch.rand((T, k), generator=gen, device="cuda")
    want, wants = B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:])
    wantx = B.moe_permute_backward(y, inv, T, k, active_rows=offsets[E:])
    part = slice(30, 60)
    few = inv.view(T, k)[part].reshape(-1).contiguous()
    dy, ds = torch.full_like(y, 7.0), torch.empty((30, k), device="cuda")
    B.moe_combine_backward(dout[part], y, few, scale[part], active_rows=offsets[E:], out=(dy, ds))
    named = torch.zeros(T * k, dtype=torch.bool, device="cuda")
    named[few.long()] = True
    assert torch.equal(dy[named], want[named]) and bool((dy[~named] == 7).all()) and torch.equal(ds, wants[part])
    assert torch.equal(B.moe_permute_backward(y, few, 30, k, active_rows=offsets[E:]), wantx[part])
    stray = inv.clone()
    stray[inv >= int(offsets[E])] = torch.tensor(2 ** 31 - 1, dtype=torch.int32, device="cuda")
    stray[:1] = -5
    dy, ds = B.moe_combine_backward(dout, y, stray, scale, active_rows=offsets[E:])
    assert float(ds.view(-1)[0]) == 0 and torch.equal(ds.view(-1)[1:], wants.view(-1)[1:])


def test_against_differences():
    """<gradient, direction> against the forward call's difference: combine is linear in y and in the scales, so a difference of two calls is exact up to rounding."""
    gen = generator(9)
    T, k, d, E = 61, 2, 256, 8
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, "pruned"), E)
    active = offsets[E:]
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    y, scale, dout, ty, ts = r(T * k, d), r(T, k), r(T, d), r(T * k, d), r(T, k)
    dy, ds = B.moe_combine_backward(dout, y, inv, scale, active_rows=active)
    f = lambda y, s: B.moe_combine(y, inv, s, T, k, active_rows=active).double()  # noqa: E731
    for got, diff in ((dy.double() * ty, f(ty, scale)), (ds.double() * ts, f(y, ts))):
        want = (dout.double() * diff).sum()
        # sums of T d products, each off by a few roundings: 16 of them of the sum of magnitudes
        assert abs(float(got.sum() - want)) <= 16 * U * float(got.abs().sum() + (dout.double() * diff).abs().sum()) + d * U * float(got.abs().sum())


def test_more_than_four_gigabytes_of_rows():
    gen = generator(1)
    T, k, d = (1 << 16) + 50, 2, 8192
    perm, inv, offsets = sorted_index(routing(gen, T, k, 4, "even"), 4)
    y = torch.empty((T * k, d), device="cuda", dtype=F32).normal_(generator=gen)
    dout, scale = torch.randn((T, d), generator=gen, device="cuda"), torch.rand((T, k), generator=gen, device="cuda")
    assert y.numel() * 4 > 1 << 32
    dy, ds = B.moe_combine_backward(dout, y, inv, scale)
    dx = B.moe_permute_backward(y, inv, T, k)
    for t in range(0, T, 8192):
        part = inv.view(T, k)[t:t + 8192].reshape(-1).contiguous()
        rows = y[part.long()]
        order = torch.arange(len(part), dtype=torch.int32, device="cuda")
        n = len(part) // k
        few, fews = B.moe_combine_backward(dout[t:t + n], rows, order, scale[t:t + n])
        assert torch.equal(dy[part.long()], few) and torch.equal(ds[t:t + n], fews) and torch.equal(dx[t:t + n], B.moe_permute_backward(rows, order, n, k)), t


def test_replays_from_a_graph_and_on_a_side_stream():
    gen = generator(2)
    T, k, d, E = 300, 2, 264, 8
    perm, inv, offsets = sorted_index(routing(gen, T, k, E, "pruned"), E)
    dout, y, scale = torch.empty((T, d), device="cuda"), torch.empty((T * k, d), dtype=F16, device="cuda"), torch.rand((T, k), generator=gen, device="cuda")
    dy, ds, dx = torch.empty_like(y), torch.empty_like(scale), torch.empty((T, d), dtype=F16, device="cuda")

    def step():
        B.moe_combine_backward(dout, y, inv, scale, active_rows=offsets[E:], out=(dy, ds))
        B.moe_permute_backward(dy, inv, T, k, active_rows=offsets[E:], out=dx)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for rep in range(4):
        dout.normal_(generator=gen)
        y.normal_(generator=gen)
        step()
        want = [t.clone() for t in (dy, ds, dx)]
        for t in (dy, ds, dx):
            t.fill_(7.0)
        torch.cuda.synchronize()
        if rep % 2:
            with torch.cuda.stream(side):
                step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dy, ds, dx), want)), rep


@pytest.mark.parametrize("T", [2 ** 22 * 4 + 5, 2 ** 31 - 1])
def test_combine_backward_of_more_tokens_than_a_launch_has_wavefronts(T):
    """The wavefronts' steps over the tokens end at T, also where T and a step together pass 2^31; every token has its dscale, the last one included."""
    need = T * (16 + 4 + 4 + 4)
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip("%d GB of memory needed" % (need >> 30))
    dout = torch.empty((T, 8), dtype=torch.float16, device="cuda").fill_(0.5)
    y = torch.full((4, 8), 2.0, dtype=torch.float16, device="cuda")
    inv = torch.empty(T, dtype=torch.int32, device="cuda").fill_(-1)
    inv[0], inv[T // 2], inv[T - 2], inv[T - 1] = 0, 1, 2, 3
    scale = torch.empty((T, 1), device="cuda").fill_(0.25)
    ds = torch.empty((T, 1), device="cuda").fill_(7.0)
    dy, _ = B.moe_combine_backward(dout, y, inv, scale, out=(torch.zeros_like(y), ds))
    torch.cuda.synchronize()
    assert bool((dy == 0.125).all())
    assert [float(ds[i]) for i in (0, T // 2, T - 2, T - 1)] == [8.0] * 4
    ends = (ds[:1 << 23], ds[-(1 << 23):])
    assert [int((t != 0).sum()) for t in ends] == [1, 2] and all(bool(((t == 0) | (t == 8)).all()) for t in ends)
    del dout, inv, scale, ds, ends
    torch.cuda.empty_cache()
