"""Low-rank adapters, forward and backward, against the formulas in 64 bits: types, odd ranks and widths, strides, rows of no adapter, orders, single tokens."""
import pytest
import torch

from paper_2211_10017_amd import binding as B
from tuning_ref import BF16, F16, F32, adapters_ref, generator, routing, sorted_index, within

pytestmark = pytest.mark.gpu
# T, k, E, K, N, rank, load
CASES = [(1, 1, 1, 8, 8, 1, "even"), (1, 1, 8, 1024, 1024, 16, "even"), (1, 2, 8, 64, 72, 3, "even"), (3, 1, 5, 16, 264, 8, "ends"), (17, 1, 3, 72, 8, 17, "even"),
         (64, 1, 32, 256, 512, 16, "pruned"), (65, 2, 130, 264, 136, 33, "even"), (128, 1, 1, 520, 64, 64, "even"), (200, 2, 16, 704, 1032, 12, "pruned"), (257, 1, 4, 128, 384, 128, "one"),
         (513, 2, 33, 136, 72, 5, "ends"), (96, 3, 7, 64, 64, 31, "pruned"), (40, 1, 6, 64, 64, 4, "none"), (1000, 1, 2, 1032, 200, 15, "one"), (700, 2, 600, 64, 128, 8, "even"),
         (2100, 1, 3, 512, 576, 32, "even"), (4100, 2, 64, 72, 64, 16, "even"), (31, 1, 4, 4104, 24, 9, "even"), (30, 1, 3, 24, 4104, 9, "even"),
         (1, 1, 3, 4096, 136, 128, "even"), (45, 2, 5, 2056, 200, 65, "pruned"), (300, 1, 7, 1032, 4104, 127, "ends")]
TYPES = [(F16, F16), (BF16, BF16), (BF16, F32), (F16, F32), (F16, BF16), (BF16, F16)]


def inputs(T, k, E, K, N, rank, load, xt, yt):
    gen = generator(T * 7 + K + rank)
    idx = routing(gen, T, k, E, load)
    perm, inv, offsets = sorted_index(idx, E)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    R = T * k
    return dict(x=r(T, K).to(xt), a=(r(E, rank, K) * K ** -0.5).to(xt), b=(r(E, rank, N) * 0.3).to(xt), scale=torch.rand(E, generator=gen, device="cuda") + 0.5, y=r(R, N).to(yt),
                dy=(r(R, N) * 0.1).to(yt), perm=perm, offsets=offsets, R=R)


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("T,k,E,K,N,rank,load", CASES)
@pytest.mark.parametrize("by_assignment", [False, True])
def test_forward_and_backward(T, k, E, K, N, rank, load, xt, yt, by_assignment):
    print(f"adapters T={T} k={k} E={E} K={K} N={N} rank={rank} {load} {xt} {yt} by_assignment={by_assignment}", flush=True)
    d = inputs(T, k, E, K, N, rank, load, xt, yt)
    index = dict(perm_src=d["perm"], k=k, scale=d["scale"], by_assignment=by_assignment)
    active = int(d["offsets"][E])
    v = torch.full((d["R"], rank), 7.0, device="cuda")
    out = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], v=v, **index)
    want = adapters_ref(d["x"], d["a"], d["b"], d["offsets"], d["perm"], k, d["scale"], by_assignment, d["y"], d["dy"])
    torch.cuda.synchronize()
    within(v[:active], want["v"][:active], (K + 4) * 2.0 ** -24 * want["v_mag"][:active])
    assert bool((v[active:] == 7).all())
    # (y itself is added with one rounding in fp32)
    within(out, want["out"], want["out_mag"] + 2.0 ** -23 * (want["out"].abs() + d["y"].double().abs()))
    inplace = d["y"].clone()
    assert B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=inplace, out=inplace, **index) is inplace
    alone = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y_dtype=yt, **index)
    torch.cuda.synchronize()
    assert torch.equal(inplace, out)
    delta = want["out"] - d["y"].double()
    within(alone, delta, want["out_mag"] + 2.0 ** -23 * delta.abs())
    dead = (d["perm"].long() if by_assignment else torch.arange(d["R"], device="cuda"))[active:]
    assert torch.equal(out[dead], d["y"][dead]) and bool((alone[dead] == 0).all())
    for kind in (xt, F32):
        dx, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], grad_dtype=kind, **index)
        torch.cuda.synchronize()
        within(dx, want["dx"], want["dx_mag"] + 2.0 ** -23 * want["dx"].abs())
        within(da, want["da"], want["da_mag"] + 2.0 ** -23 * want["da"].abs())
        within(db, want["db"], want["db_mag"] + 2.0 ** -23 * want["db"].abs())
        assert da.dtype == kind and bool((dx[dead] == 0).all())
        empty = d["offsets"][1:] == d["offsets"][:-1]
        assert bool((da[empty] == 0).all()) and bool((db[empty] == 0).all())


@pytest.mark.parametrize("xt,yt", [(F16, F16), (BF16, F32)])
@pytest.mark.parametrize("T,E,K,N,rank", [(1, 1, 64, 64, 4), (90, 1, 128, 264, 8), (600, 5, 72, 64, 16)])
def test_rows_that_are_sorted_already(T, E, K, N, rank, xt, yt):
    """Without perm_src: x's rows in the order of the adapters, here with more rows than the offsets say; scale 1 without one."""
    d = inputs(T, 1, E, K, N, rank, "even", xt, yt)
    offsets = torch.linspace(0, T - T // 10, E + 1, device="cuda").int()
    v = torch.zeros((T, rank), device="cuda")
    out = B.moe_adapters(d["x"], d["a"], d["b"], offsets, y=d["y"], v=v)
    dx, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, offsets)
    want = adapters_ref(d["x"], d["a"], d["b"], offsets, None, 1, None, False, d["y"], d["dy"])
    torch.cuda.synchronize()
    within(out, want["out"], want["out_mag"] + 2.0 ** -23 * (want["out"].abs() + d["y"].double().abs()))
    for got, name in ((dx, "dx"), (da, "da"), (db, "db")):
        within(got, want[name], want[name + "_mag"] + 2.0 ** -23 * want[name].abs())


@pytest.mark.parametrize("T,E,K,N,rank", [(1, 4, 64, 64, 4), (77, 6, 264, 136, 12), (600, 3, 128, 512, 16)])
def test_slices_of_wider_rows(T, E, K, N, rank):
    """x, y, out, dy and dx as columns of wider matrices: what is beside them stays, and the results are those of whole ones."""
    d = inputs(T, 1, E, K, N, rank, "pruned", BF16, BF16)
    wide = lambda t: torch.full((t.shape[0], t.shape[1] + 24), 3.0, dtype=t.dtype, device="cuda")  # noqa: E731
    inner = lambda t: t[:, 8:8 + t.shape[1] - 24]  # noqa: E731
    put = lambda t: (lambda w: (inner(w).copy_(t), w)[1])(wide(t))  # noqa: E731
    index = dict(perm_src=d["perm"], scale=d["scale"], by_assignment=True)
    x, y, dy, out, dx = put(d["x"]), put(d["y"]), put(d["dy"]), wide(d["y"]), wide(d["x"])
    v = torch.empty((T, rank), device="cuda")
    B.moe_adapters(inner(x), d["a"], d["b"], d["offsets"], y=inner(y), out=inner(out), v=v, **index)
    B.moe_adapters_backward(inner(dy), inner(x), d["a"], d["b"], v, d["offsets"], out=(inner(dx), None, None), need=(True, False, False), **index)
    B.moe_adapters(inner(x), d["a"], d["b"], d["offsets"], y=inner(y), out=inner(y), **index)
    w = torch.empty_like(v)
    want = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], v=w, **index)
    wants = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], w, d["offsets"], **index)
    torch.cuda.synchronize()
    assert torch.equal(inner(out), want) and torch.equal(inner(y), want) and torch.equal(inner(dx), wants[0])
    for t in (out, y, dx):
        assert bool((t[:, :8] == 3).all()) and bool((t[:, t.shape[1] - 16:] == 3).all())


def test_offsets_that_are_no_partition_stay_inside():
    """Wrong results, but nothing behind the buffers: the canaries around them stay."""
    T, E, K, N, rank = 3000, 9, 64, 128, 16
    d = inputs(T, 1, E, K, N, rank, "even", BF16, BF16)
    need = B.moe_adapters_backward_workspace_bytes(T, E, K, N, rank)
    for offsets in ([0, T] * 5, [T, 0] * 5, [-5, 10 ** 9] * 5, [2 ** 31 - 1] * 10, [0, 2500, 100, 2900, 0, 3000, 0, 3000, 10, 3000]):
        off = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
        guarded = {}

        def guard(name, n, dtype):
            t = torch.full((n + 1024,), 7.0, dtype=dtype, device="cuda")
            guarded[name] = t
            return t[512:512 + n]

        out, v = guard("out", T * N, BF16).view(T, N), guard("v", T * rank, F32).view(T, rank)
        grads = guard("dx", T * K, BF16).view(T, K), guard("da", E * rank * K, F32).view(E, rank, K), guard("db", E * rank * N, F32).view(E, rank, N)
        B.moe_adapters(d["x"], d["a"], d["b"], off, y=d["y"], out=out, v=v, perm_src=d["perm"], by_assignment=True)
        v.nan_to_num_(0.0)
        B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, off, perm_src=d["perm"], out=grads, workspace=ws[:need])
        torch.cuda.synchronize()
        assert bool((ws[need:] == 77).all())
        for name, t in guarded.items():
            assert bool((t[:512] == 7).all()) and bool((t[-512:] == 7).all()), name


def test_needs_one_by_one_and_repeats():
    """Each gradient alone has the bits of all together; the same call has the same bits."""
    d = inputs(300, 2, 8, 264, 136, 16, "pruned", F16, F16)
    index = dict(perm_src=d["perm"], k=2, scale=d["scale"])
    v = torch.empty((600, 16), device="cuda")
    out = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], v=v, **index)
    assert torch.equal(B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], **index), out)
    every = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], **index)
    for i in range(3):
        need = tuple(j == i for j in range(3))
        got = B.moe_adapters_backward(d["dy"], d["x"] if i == 1 else None, d["a"], d["b"], v if i == 2 else None, d["offsets"], need=need, **index)
        assert torch.equal(got[i], every[i]) and all(got[j] is None for j in range(3) if j != i)


def test_other_rows_do_not_reach_a_row():
    """An infinity or a NaN in the rows of one adapter, or of none, stays there."""
    T, E, K, N, rank = 200, 5, 136, 72, 12
    for xt, yt in ((BF16, F32), (F16, F16)):
        d = inputs(T, 1, E, K, N, rank, "pruned", xt, yt)
        index = dict(perm_src=d["perm"], scale=d["scale"], by_assignment=True)
        v = torch.empty((T, rank), device="cuda")
        want = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], v=v, **index)
        wants = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], **index)
        off = d["offsets"].tolist()
        bad = torch.cat([d["perm"][off[2]:off[3]], d["perm"][off[E]:]]).long()
        fine = torch.ones(T, dtype=torch.bool, device="cuda")
        fine[bad] = False
        x, dy = d["x"].clone(), d["dy"].clone()
        x[bad[::2]], x[bad[1::2]], dy[bad] = float("nan"), float("inf"), float("nan")
        w = torch.empty_like(v)
        got = B.moe_adapters(x, d["a"], d["b"], d["offsets"], y=d["y"], v=w, **index)
        gots = B.moe_adapters_backward(dy, x, d["a"], d["b"], w, d["offsets"], **index)
        torch.cuda.synchronize()
        assert torch.equal(got[fine], want[fine]) and torch.equal(gots[0][fine], wants[0][fine])
        for g, o in zip(gots[1:], wants[1:]):
            assert all(torch.equal(g[e], o[e]) for e in range(E) if e != 2) and bool(torch.isnan(g[2]).any())


@pytest.mark.parametrize("xt", [F16, BF16])
@pytest.mark.parametrize("size", [2.0 ** -40, 2.0 ** 20])
def test_rows_of_any_size(xt, size):
    """Gradients far below what 16 bits hold, and coefficients far above: v and u are fp32 numbers."""
    T, E, K, N, rank = 150, 4, 256, 128, 16
    d = inputs(T, 1, E, K, N, rank, "even", xt, F32)
    d["dy"] = d["dy"] * size
    scale = d["scale"] * size
    index = dict(perm_src=d["perm"], k=1)
    v = torch.empty((T, rank), device="cuda")
    out = B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=None, y_dtype=F32, v=v, scale=scale, **index)
    want = adapters_ref(d["x"], d["a"], d["b"], d["offsets"], d["perm"], 1, scale, False, None, d["dy"])
    within(out, want["out"], want["out_mag"] + 2.0 ** -23 * want["out"].abs())
    dx, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], grad_dtype=F32, scale=d["scale"], **index)
    want = adapters_ref(d["x"], d["a"], d["b"], d["offsets"], d["perm"], 1, d["scale"], False, None, d["dy"])
    torch.cuda.synchronize()
    if xt == BF16:
        within(dx, want["dx"], want["dx_mag"] + 2.0 ** -23 * want["dx"].abs())
    within(da, want["da"], want["da_mag"] + 2.0 ** -23 * want["da"].abs())
    within(db, want["db"], want["db_mag"] + 2.0 ** -23 * want["db"].abs())


def test_against_differences():
    """The gradient along random directions against central differences of the forward call in fp32: out is linear in x, a and b each, so a difference of two calls has no error but roundings."""
    T, E, K, N, rank = 50, 3, 64, 72, 8
    d = inputs(T, 1, E, K, N, rank, "pruned", BF16, F32)
    gen = generator(77)
    index = dict(perm_src=d["perm"], scale=d["scale"], by_assignment=True)
    v = torch.empty((T, rank), device="cuda")
    f = lambda x, a, b: B.moe_adapters(x, a, b, d["offsets"], y_dtype=F32, v=v, **index).double()  # noqa: E731
    f(d["x"], d["a"], d["b"])
    grads = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], grad_dtype=F32, **index)
    v = v.clone()
    for i, name in enumerate(("x", "a", "b")):
        t = torch.randn(d[name].shape, generator=gen, device="cuda").to(BF16)
        args = [d["x"], d["a"], d["b"]]
        args[i] = t
        along = (d["dy"].double() * f(*args)).sum()
        got = grads[i].double() * t.double()
        # dx is rounded to bf16, 2^-8 of each term; the sums otherwise by 2^-16 of theirs and fp32's roundings
        rounding = 2.0 ** -8 if name == "x" else 2.0 ** -14
        assert abs(float(got.sum() - along)) <= rounding * float(got.abs().sum()) + 2.0 ** -14 * float((d["dy"].double() * f(*args)).abs().sum())


def test_replays_from_a_graph_and_on_a_side_stream():
    T, k, E, K, N, rank = 120, 2, 6, 264, 136, 16
    d = inputs(T, k, E, K, N, rank, "pruned", F16, F16)
    gen = generator(4)
    index = dict(perm_src=d["perm"], k=k, scale=d["scale"])
    v, out = torch.empty((d["R"], rank), device="cuda"), torch.empty_like(d["y"])
    ws = torch.empty(B.moe_adapters_backward_workspace_bytes(d["R"], E, K, N, rank), dtype=torch.uint8, device="cuda")
    grads = torch.empty((d["R"], K), dtype=F16, device="cuda"), torch.empty_like(d["a"]), torch.empty_like(d["b"])

    def step():
        B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], out=out, v=v, **index)
        B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], out=grads, workspace=ws, **index)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for rep in range(4):
        d["x"].normal_(generator=gen)
        d["y"].normal_(generator=gen)
        d["dy"].normal_(generator=gen)
        step()
        results = (out, *grads)
        want = [t.clone() for t in results]
        for t in results:
            t.fill_(7.0)
        torch.cuda.synchronize()
        if rep % 2:
            with torch.cuda.stream(side):
                step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(results, want)), rep


@pytest.mark.parametrize("R,E", [(256, 1), (511, 1), (512, 1), (700, 2), (768, 2), (1024, 3), (1024, 4), (1025, 4)])
def test_gradients_of_few_adapters_with_all_the_rows(R, E):
    """One part of an adapter's rows or several, around where that changes; the last adapter has every row, the others' gradients are 0."""
    K, N, rank = 72, 136, 8
    d = inputs(R, 1, E, K, N, rank, "even", BF16, BF16)
    off = torch.tensor([0] * E + [R], dtype=torch.int32, device="cuda")
    index = dict(perm_src=d["perm"], scale=d["scale"], by_assignment=True)
    v = torch.empty((R, rank), device="cuda")
    B.moe_adapters(d["x"], d["a"], d["b"], off, y=d["y"], v=v, **index)
    want = adapters_ref(d["x"], d["a"], d["b"], off, d["perm"], 1, d["scale"], True, d["y"], d["dy"])
    _, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, off, **index)
    torch.cuda.synchronize()
    within(da, want["da"], want["da_mag"] + 2.0 ** -23 * want["da"].abs())
    within(db, want["db"], want["db_mag"] + 2.0 ** -23 * want["db"].abs())
    assert bool((da[:-1] == 0).all()) and bool((db[:-1] == 0).all())


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("T,rank", [(3400, 50), (7000, 64), (8200, 33), (11800, 61), (3400, 127), (9000, 100), (10100, 128)])
def test_blocks_of_a_high_rank(T, rank, xt, yt):
    """Shares of rows that fill blocks of 32, 48 and 64 rows, with ranks above 32."""
    test_forward_and_backward(T, 1, 5, 72, 136, rank, "even", xt, yt, True)


@pytest.mark.parametrize("T,rank", [(3400, 16), (3400, 50), (8000, 60), (9000, 100)])
def test_gradient_of_a_alone(T, rank):
    """Coefficients that are wanted by themselves, in blocks of more than sixteen rows."""
    d = inputs(T, 1, 5, 72, 136, rank, "pruned", BF16, F32)
    index = dict(perm_src=d["perm"], scale=d["scale"], by_assignment=True)
    want = adapters_ref(d["x"], d["a"], d["b"], d["offsets"], d["perm"], 1, d["scale"], True, d["y"], d["dy"])
    dx, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], None, d["offsets"], need=(False, True, False), **index)
    torch.cuda.synchronize()
    assert dx is None and db is None
    within(da, want["da"], want["da_mag"] + 2.0 ** -23 * want["da"].abs())


@pytest.mark.parametrize("E", range(1, 10))
def test_one_matrix_of_any_number_of_adapters(E):
    """The grid is rounded up to whole rounds of the eight XCDs: what is left over belongs to neither matrix, also where one of them is not wanted."""
    d = inputs(40, 1, E, 64, 64, 8, "even", F16, F16)
    index = dict(perm_src=d["perm"], scale=d["scale"])
    v = torch.empty((40, 8), device="cuda")
    B.moe_adapters(d["x"], d["a"], d["b"], d["offsets"], y=d["y"], v=v, **index)
    _, da, db = B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], v, d["offsets"], **index)
    for kept in (v, None):
        assert torch.equal(B.moe_adapters_backward(d["dy"], d["x"], d["a"], d["b"], kept, d["offsets"], need=(False, True, False), **index)[1], da)
    assert torch.equal(B.moe_adapters_backward(d["dy"], None, d["a"], d["b"], v, d["offsets"], need=(False, False, True), **index)[2], db)
