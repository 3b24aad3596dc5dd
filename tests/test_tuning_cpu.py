"""What the calls that layers are tuned with refuse on the host, before anything is launched: the exchange's gradient, adapters, AdamW."""
import ctypes

import pytest
import torch

from launches import P as PTR, record
from paper_2211_10017_amd import AdamW, LowRankAdapters, adapt
from paper_2211_10017_amd import combine_tokens, permute_tokens
from paper_2211_10017_amd import binding as B

P, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)          # never dereferenced: validation fails first
OK, ARG, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
F16, BF16, F32 = 0, 1, 2
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    return B.load()


def test_exchange_refusals(lib):
    def combine(dout=P, odt=F32, y=P, ydt=F16, inv=P, scale=P, T=4, k=2, d=64, R=8, dy=P, ds=P):
        return lib.moe_combine_backward(dout, odt, y, ydt, inv, scale, None, T, k, d, R, dy, ds, None)

    def permute(g=P, gdt=F16, inv=P, T=4, k=2, d=64, R=8, dx=P, dt=F32):
        return lib.moe_permute_backward(g, gdt, inv, None, T, k, d, R, dx, dt, None)

    for name in ("dout", "y", "inv", "scale"):
        assert combine(**{name: None}) == ARG and b"NULL" in lib.moe_last_error(), name
    assert combine(dy=None, ds=None) == ARG and combine(dy=None, y=None) == ARG
    for name in ("dout", "y", "dy"):
        assert combine(**{name: ODD}) == ARG and b"aligned" in lib.moe_last_error(), name
    for name in ("g", "inv", "dx"):
        assert permute(**{name: None}) == ARG and b"NULL" in lib.moe_last_error(), name
    for name in ("g", "dx"):
        assert permute(**{name: ODD}) == ARG, name
    for call in (combine, permute):
        for bad in (dict(T=-1), dict(k=0), dict(d=0), dict(d=60), dict(R=-1), dict(T=2 ** 30, k=2)):
            assert call(**bad) == ARG, bad
        assert call(T=0, inv=None) == OK                            # empty buffers may be NULL
    assert combine(odt=3) == UNSUPPORTED and combine(ydt=-1) == UNSUPPORTED and permute(gdt=3) == UNSUPPORTED and permute(dt=7) == UNSUPPORTED


def _adapters(lib, x=P, dt=F16, xs=64, T=4, perm=P, k=2, off=P, R=8, E=3, K=64, N=72, rank=8, a=P, b=P, by=0, y=P, ys=72, out=P, os=72, ydt=F16, v=P):
    return lib.moe_adapters(x, dt, xs, T, perm, k, off, R, E, K, N, rank, a, b, P, by, y, ys, out, os, ydt, v, None)


def _backward(lib, dy=P, ydt=F16, dys=72, x=P, dt=F16, xs=64, T=4, perm=P, k=2, off=P, R=8, E=3, K=64, N=72, rank=8, a=P, b=P, by=0, v=P, dx=P, dxs=64, da=P, db=P, gdt=F32, ws=P,
              size=1 << 40):
    return lib.moe_adapters_backward(dy, ydt, dys, x, dt, xs, T, perm, k, off, R, E, K, N, rank, a, b, P, by, v, dx, dxs, da, db, gdt, ws, size, None)


def test_adapter_refusals(lib):
    for call in (_adapters, _backward):
        for bad in (dict(T=-1), dict(R=-1), dict(k=0), dict(E=0), dict(K=0), dict(N=-8), dict(K=60, xs=60), dict(N=68), dict(rank=0), dict(R=7), dict(T=5), dict(perm=None), dict(off=None),
                    dict(a=None), dict(b=None), dict(a=ODD), dict(b=ODD), dict(x=None), dict(x=ODD), dict(xs=56), dict(xs=68), dict(perm=None, k=1, by=1, R=4)):
            assert call(lib, **bad) == ARG, (call.__name__, bad, lib.moe_last_error())
        for bad in (dict(rank=129), dict(E=4097), dict(dt=F32), dict(ydt=4), dict(K=2 ** 20 + 8, xs=2 ** 20 + 8)):
            assert call(lib, **bad) == UNSUPPORTED, (call.__name__, bad)
    assert _adapters(lib, v=ODD) == ARG and _adapters(lib, v=None, R=514, T=257, y=ODD) == ARG and _adapters(lib, v=None, R=514, T=257) == ARG and b"NULL" in lib.moe_last_error()
    for bad in (dict(y=ODD), dict(out=ODD), dict(out=None), dict(ys=64), dict(os=64), dict(ys=76), dict(ys=80)):      # (the last: in place with two strides)
        assert _adapters(lib, **bad) == ARG, bad
    for bad in (dict(dy=None), dict(dy=ODD), dict(dys=64), dict(v=None), dict(v=ODD), dict(ws=ODD), dict(dx=ODD), dict(dxs=56), dict(da=ODD), dict(db=ODD)):
        assert _backward(lib, **bad) == ARG, bad
    assert _backward(lib, gdt=3) == UNSUPPORTED
    assert _backward(lib, ws=None) == WORKSPACE and _backward(lib, size=15) == WORKSPACE and b"workspace" in lib.moe_last_error()
    assert _adapters(lib, T=0, R=0, x=None, y=None, out=None, perm=P) == OK


def test_adapter_workspaces(lib):
    q = lib.moe_adapters_backward_workspace_bytes
    assert q(0, 4, 64, 64, 8) == 0 and q(8, 0, 64, 64, 8) == 0
    assert q(100, 4, 64, 64, 8) >= 100 * 8 * 4
    need = q(8, 3, 64, 72, 8)
    assert _backward(lib, size=need - 1) == WORKSPACE


class Tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "g", "m", "v", "ms", "vs", "copy")] + [("n", ctypes.c_int64)]


def test_adamw_refusals(lib):
    def call(count=1, pd=F32, gd=F32, cd=-1, bits=32, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, wd=0.0, gs=1.0, step=1, table=None, **fields):
        t = Tensor(*[0x1000] * 7, 64)
        for name, value in fields.items():
            setattr(t, name, value)
        return lib.moe_adamw(ctypes.byref(t) if table is None else table, count, pd, gd, cd, bits, lr, b1, b2, eps, wd, gs, step, None, None)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(count=-1), dict(step=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(eps=-1e-8), dict(eps=inf), dict(wd=-1.0),
                dict(gs=inf), dict(gs=nan), dict(n=-1), dict(p=0), dict(g=0), dict(m=0), dict(v=0), dict(bits=8, ms=0), dict(bits=8, vs=0), dict(cd=F16, copy=0), dict(p=0x1002),
                dict(g=0x1001, gd=F16), dict(m=0x1002), dict(cd=BF16, copy=0x1001)):
        assert call(**bad) == ARG, bad
    for bad in (dict(pd=3), dict(gd=-1), dict(cd=F32), dict(cd=F16, pd=BF16), dict(bits=16), dict(n=2 ** 40)):
        assert call(**bad) == UNSUPPORTED, bad
    assert lib.moe_adamw(None, 1, F32, F32, -1, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0, 1, None, None) == ARG
    assert lib.moe_adamw(None, 0, F32, F32, -1, 32, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0, 1, None, None) == OK and call(n=0, p=0) == OK
    state = lambda codes=P, scales=P, n=64, out=P, dt=F32: lib.moe_adamw_state(codes, scales, n, out, dt, None)  # noqa: E731
    assert state(n=-1) == ARG and state(codes=None) == ARG and state(scales=None) == ARG and state(out=None) == ARG and state(out=ctypes.c_void_p(0x1002)) == ARG
    assert state(dt=5) == UNSUPPORTED and state(n=0, codes=None) == OK


@pytest.fixture
def on_host(monkeypatch):
    """The binding with a library that takes every call, on tensors of the CPU."""
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: called.append(name) or 0

    monkeypatch.setattr(B, "load", lambda: Library())
    monkeypatch.setattr(B, "_stream", lambda: 0)
    monkeypatch.setattr(B, "_raw_device", lambda: -1)                # (where a tensor of the CPU says it is)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    return called


def test_binding_refuses_shapes_that_do_not_fit(on_host):
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    h, i32 = torch.float16, torch.int32
    T, k, d, R = 4, 2, 64, 8
    combine = dict(dout=z(T, d), y_perm=z(R, d, dt=h), inv_perm=z(R, dt=i32), expert_scale=z(T, k))
    B.moe_combine_backward(**combine)
    for bad in (dict(dout=z(T, d + 8)), dict(dout=z(T + 1, d)), dict(dout=z(T, 2 * d)[:, ::2]), dict(inv_perm=z(R - 1, dt=i32)), dict(inv_perm=z(R)), dict(expert_scale=z(T, k, dt=h)),
                dict(expert_scale=z(R)), dict(y_perm=z(R, d, dt=i32)), dict(out=(z(R, d), z(T, k))), dict(out=(z(R - 1, d, dt=h), z(T, k))), dict(active_rows=z(0, dt=i32))):
        with pytest.raises(B.MoeError):
            B.moe_combine_backward(**dict(combine, **bad))
    B.moe_permute_backward(z(R, d), z(R, dt=i32), T, k)
    for bad in ((z(R * d), z(R, dt=i32), T, k), (z(R, d), z(R, dt=i32), T + 1, k), (z(R, d), z(R), T, k)):
        with pytest.raises(B.MoeError):
            B.moe_permute_backward(*bad)
    with pytest.raises(B.MoeError):
        B.moe_permute_backward(z(R, d), z(R, dt=i32), T, k, out=z(T, d + 8))
    E, rank, K, N = 3, 8, 64, 72
    make = lambda: dict(x=z(T, K, dt=h), a=z(E, rank, K, dt=h), b=z(E, rank, N, dt=h), expert_offsets=z(E + 1, dt=i32), perm_src=z(R, dt=i32), k=k, scale=z(E), y=z(R, N), out=z(R, N),  # noqa: E731
                        v=z(R, rank))
    B.moe_adapters(**make())
    B.moe_adapters(**dict(make(), x=z(T, 2 * K, dt=h)[:, K:]))         # a slice of wider rows
    for bad in (dict(x=z(T, K)), dict(x=z(T, K + 8, dt=h)), dict(x=z(T, 2 * K, dt=h)[:, ::2]), dict(a=z(E, rank, K)), dict(b=z(E, rank + 1, N, dt=h)), dict(b=z(E, rank, N, dt=torch.bfloat16)),
                dict(expert_offsets=z(E, dt=i32)), dict(scale=z(E + 1)), dict(scale=z(E, dt=h)), dict(perm_src=z(R)), dict(perm_src=None), dict(y=z(R - 1, N)), dict(y=z(R, N, dt=h)),
                dict(out=z(R + 1, N)), dict(out=z(R, N, dt=i32)), dict(v=z(R, rank + 1)), dict(v=z(R, rank, dt=h)), dict(a=z(E * rank, K, dt=h))):
        with pytest.raises(B.MoeError):
            B.moe_adapters(**dict(make(), **bad))
    back = lambda: dict(dy=z(R, N), x=z(T, K, dt=h), a=z(E, rank, K, dt=h), b=z(E, rank, N, dt=h), v=z(R, rank), expert_offsets=z(E + 1, dt=i32), perm_src=z(R, dt=i32), k=k,  # noqa: E731
                        workspace=z(4096, dt=torch.uint8))
    B.moe_adapters_backward(**back())
    for bad in (dict(dy=z(R + 1, N)), dict(dy=z(R, N, dt=i32)), dict(x=None), dict(v=None), dict(v=z(R, rank, dt=h)), dict(x=z(T, K)), dict(out=(z(R, K), None, None)),
                dict(out=(None, z(E, rank, K), z(E, rank, N, dt=h))), dict(out=(None, z(E, rank, K + 8), None))):
        with pytest.raises(B.MoeError):
            B.moe_adapters_backward(**dict(back(), **bad))


def test_binding_refuses_lists_that_do_not_fit(on_host):
    z = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt)  # noqa: E731
    u8 = torch.uint8
    make = lambda: [[z(40), z(3)], [z(40), z(3)], [z(40), z(3)], [z(40), z(3)], 1]  # noqa: E731
    B.moe_adamw(*make())
    B.moe_adamw([], [], [], [], 1)
    with pytest.raises(B.MoeError, match="twice"):
        p = z(40)
        B.moe_adamw([p, p], [z(40), z(40)], [z(40), z(40)], [z(40), z(40)], 1)
    for at, value in ((0, [z(40)]), (1, [z(40), z(4)]), (1, [z(40), z(3, torch.float16)]), (2, [z(40), z(3, torch.float16)]), (3, [z(41), z(3)]), (0, [z(40), z(3, torch.float64)]),
                      (1, [z(80)[::2], z(3)]), (4, z(2, torch.int32)), (4, z(1)), (2, [(z(40, u8), z(2, u8))] * 2)):
        args = make()
        args[at] = value
        with pytest.raises((B.MoeError, ValueError, TypeError)):
            B.moe_adamw(*args)
    eight = lambda: [(z(40, u8), z(2, u8)), (z(3, u8), z(1, u8))]  # noqa: E731
    B.moe_adamw([z(40), z(3)], [z(40), z(3)], eight(), eight(), 1, copies=[z(40, torch.float16), z(3, torch.float16)])
    for m in ([(z(40, u8), z(1, u8)), (z(3, u8), z(1, u8))], [(z(39, u8), z(2, u8)), (z(3, u8), z(1, u8))], [(z(40), z(2, u8)), (z(3, u8), z(1, u8))]):
        with pytest.raises(B.MoeError):
            B.moe_adamw([z(40), z(3)], [z(40), z(3)], m, eight(), 1)
    for copies in ([z(40, torch.float16)], [z(40, torch.float16), z(4, torch.float16)], [z(40), z(3)], [z(40, torch.float16), z(3, torch.bfloat16)]):
        with pytest.raises(B.MoeError):
            B.moe_adamw([z(40), z(3)], [z(40), z(3)], eight(), eight(), 1, copies=copies)
    with pytest.raises(B.MoeError):
        B.moe_adamw_state(z(40, u8), z(1, u8))


def test_binding_refuses_another_device(on_host, monkeypatch):
    monkeypatch.setattr(B, "_raw_device", lambda: 1)
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    i32 = torch.int32
    for call in (lambda: B.moe_combine_backward(z(2, 8), z(2, 8), z(2, dt=i32), z(2, 1)), lambda: B.moe_permute_backward(z(2, 8), z(2, dt=i32), 2, 1),
                 lambda: B.moe_adapters(z(2, 8, dt=torch.float16), z(1, 4, 8, dt=torch.float16), z(1, 4, 8, dt=torch.float16), z(2, dt=i32)),
                 lambda: B.moe_adamw([z(4)], [z(4)], [z(4)], [z(4)], 1), lambda: B.moe_adamw_state(z(4, dt=torch.uint8), z(1, dt=torch.uint8))):
        with pytest.raises(B.MoeError, match="device"):
            call()
    assert not [name for name in on_host if not name.endswith("bytes")]


def test_the_largest_batches_take_a_launch():
    for T, d in ((1, 8), (2 ** 30, 8192)):
        for call in (("moe_combine_backward", [PTR, F32, PTR, F16, PTR, PTR, None, T, 1, d, T, PTR, PTR, None]), ("moe_permute_backward", [PTR, F16, PTR, None, T, 1, d, T, PTR, F16, None])):
            got = record([call])[0]
            assert got.rc == OK and len(got.launches) == 1 and 0 < got.launches[0].grid[0] * got.launches[0].block < 2 ** 32


X, DX = 1 << 40, 1 << 41                                             # buffers of their own


def _calls(T, k, E, K, N, rank, dt=F16, ydt=F16, v=PTR, y=PTR, out=PTR):
    R = T * k
    forward = ("moe_adapters", [X, dt, [K], T, PTR, k, PTR, R, E, K, N, rank, PTR, PTR, None, 0, y, [N], out, [N], ydt, v, None])
    backward = ("moe_adapters_backward", [PTR, ydt, [N], PTR, dt, [K], T, PTR, k, PTR, R, E, K, N, rank, PTR, PTR, None, 0, PTR, DX, [K], PTR, PTR, F32, PTR, [1 << 40], None])
    return forward, backward


def test_what_adapters_launch():
    """One launch from rows to rows but for long matrices of a high rank; gradients of the matrices another, and a third where an adapter may have more than one part."""
    sizes = {(1, 1, 8, 1024, 1024, 16): (1, 2), (64, 1, 32, 1024, 4096, 16): (1, 2), (512, 2, 16, 256, 256, 8): (1, 2), (513, 2, 16, 256, 256, 8): (1, 3), (1, 1, 8, 4096, 4096, 64): (2, 3),
             (1, 1, 8, 1024, 1024, 128): (2, 3), (1, 1, 8, 1016, 1016, 128): (1, 2), (16384, 1, 32, 4096, 4096, 32): (1, 3), (8192, 2, 64, 4096, 4096, 16): (1, 3), (16384, 1, 32, 4096, 4096, 128): (1, 3)}
    calls = [c for s in sizes for c in _calls(*s)]
    got = record(calls)
    for i, (size, (one, two)) in enumerate(sizes.items()):
        for call, want in zip(got[2 * i:2 * i + 2], (one, two)):
            assert call.rc == OK and len(call.launches) == want, (size, call)
            assert all(0 < l.grid[0] * l.block < 2 ** 32 and l.shared <= 160 * 1024 for l in call.launches)
    # without a place for the coefficients one launch keeps them on chip
    assert len(record([_calls(1, 1, 8, 4096, 4096, 128, v=None)[0]])[0].launches) == 1
    # rows of no adapter: blocks of their own, not in place (there y and out are one pointer)
    in_place, apart = record([_calls(64, 1, 32, 1024, 1024, 16)[0], _calls(64, 1, 32, 1024, 1024, 16, y=None)[0]])
    assert apart.launches[0].grid[0] == in_place.launches[0].grid[0] + 4


def test_the_most_rows_and_adapters():
    big = record([_calls(2 ** 24, 1, 4096, 64, 64, 16)[0], _calls(2 ** 24, 1, 4096, 64, 64, 16)[1], _calls(1, 1, 4096, 2 ** 20, 2 ** 20, 128)[0]])
    assert all(c.rc == OK for c in big)
    assert record([_calls(2 ** 31 - 1, 1, 1, 64, 64, 16)[0]])[0].rc in (OK, UNSUPPORTED)


def test_objects_refuse_what_calls_would():
    for bad in (dict(E=0), dict(rank=129), dict(K=60), dict(N=0), dict(dtype=torch.float32), dict(E=5000)):
        with pytest.raises(B.MoeError):
            LowRankAdapters(**dict(dict(E=2, rank=4, K=64, N=64, device="cpu"), **bad))
    a = LowRankAdapters(2, 4, 64, 72, alpha=8, device="cpu")
    assert a.a.shape == (2, 4, 64) and a.b.shape == (2, 4, 72) and bool((a.b == 0).all()) and a.scale.tolist() == [2.0, 2.0]
    p = torch.zeros(4, requires_grad=True)
    for bad in (dict(params=[]), dict(params=[p, p]), dict(params=[p], bits=16), dict(params=[torch.zeros(4, dtype=torch.float64)]), dict(params=[torch.zeros(4, 4)[:, 0]])):
        with pytest.raises(B.MoeError):
            AdamW(**bad)
    one = AdamW([p])
    with pytest.raises(B.MoeError):
        one.load_state_dict(AdamW([torch.zeros(5)]).state_dict())
    with pytest.raises(B.MoeError):
        one.load_state_dict(AdamW([p], bits=8).state_dict())
    with pytest.raises(B.MoeError, match="scale"):
        adapt(None, None, a.a, a.b, None, a.scale.requires_grad_())


def test_adapters_of_no_rows_take_null_buffers():
    """An empty batch's buffers are NULL, its index too, whatever k and the order are; gradients of the matrices are still written (as 0)."""
    calls = []
    for k, by_assignment in ((1, 0), (1, 1), (2, 0), (2, 1)):
        calls += [("moe_adapters", [None, F16, [64], 0, None, k, PTR, 0, 4, 64, 64, 4, PTR, PTR, None, by_assignment, None, [64], None, [64], F16, None, None]),
                  ("moe_adapters_backward", [None, F16, [64], None, F16, [64], 0, None, k, PTR, 0, 4, 64, 64, 4, PTR, PTR, None, by_assignment, None, None, [64], PTR, PTR, F32, None, [0], None])]
    got = record(calls)
    assert [c.rc for c in got] == [OK] * len(calls) and [len(c.launches) for c in got] == [0, 1] * (len(calls) // 2)


def test_adapters_refuse_to_write_what_they_read():
    forward, backward = _calls(64, 1, 4, 64, 64, 8)
    at = lambda call, **new: (call[0], [new.get("i%d" % i, a) for i, a in enumerate(call[1])])  # noqa: E731
    assert forward[1][0] == X and forward[1][18] == PTR and [backward[1][i] for i in (0, 3, 20)] == [PTR, PTR, DX]
    calls = [forward, backward, at(forward, i0=PTR), at(backward, i20=PTR), at(backward, i0=X, i20=X), at(backward, i3=DX), at(backward, i20=None)]
    assert [c.rc for c in record(calls)] == [OK, OK, ARG, ARG, ARG, ARG, OK]


def test_a_refused_gradient_is_no_step():
    p = torch.zeros((4, 2), requires_grad=True)
    one = AdamW([p])
    p.grad = torch.zeros((4, 2)).to_sparse()
    with pytest.raises(B.MoeError, match="dense"):
        one.step()
    assert one.steps == 0


def test_how_states_are_rounded(lib, on_host, monkeypatch):
    """The binding asks for rounding by chance where it is wanted, and AdamW with states in 8 bits wants it."""
    asked = []
    monkeypatch.setattr(B, "load", lambda: type("Library", (), {"moe_adamw": staticmethod(lambda *args: asked.append(args[5]) or 0)}))
    z, u8 = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt), torch.uint8  # noqa: E731
    eight = lambda: [(z(40, u8), z(2, u8))]  # noqa: E731
    for kw, states in ((dict(), eight), (dict(rounding="random"), eight), (dict(rounding="random"), lambda: [z(40)])):
        B.moe_adamw([z(40)], [z(40)], states(), states(), 1, **kw)
    with pytest.raises(B.MoeError, match="rounding"):
        B.moe_adamw([z(40)], [z(40)], eight(), eight(), 1, rounding="up")
    for bits in (8, 32):
        p = z(40).requires_grad_()
        p.grad = z(40)
        AdamW([p], bits=bits).step()
    assert asked == [8, 8 | B.MOE_ADAMW_RANDOM, 32, 8 | B.MOE_ADAMW_RANDOM, 32]
    t = Tensor(*[0x1000] * 7, 64)
    for bits in (32 | B.MOE_ADAMW_RANDOM, B.MOE_ADAMW_RANDOM, 9):
        assert lib.moe_adamw(ctypes.byref(t), 1, F32, F32, -1, bits, 1e-3, 0.9, 0.99, 1e-8, 0.0, 1.0, 1, None, None) == UNSUPPORTED


def test_combine_keeps_scales_that_carry_no_gradient(on_host, monkeypatch):
    """The scales that its backward pass uses are a copy (a layer's gate writes its own again through a pointer), the program's own where they learn."""
    used = []
    library = type("Library", (), {"moe_combine": staticmethod(lambda *args: 0), "moe_combine_backward": staticmethod(lambda *args: used.append(args[5]) or 0)})
    monkeypatch.setattr(B, "load", lambda: library)
    for learns in (False, True):
        y, scale = torch.zeros(8, 64).requires_grad_(), torch.ones(4, 2).requires_grad_(learns)
        combine_tokens(y, torch.arange(8, dtype=torch.int32), scale).sum().backward()
        assert (used.pop() == scale.data_ptr()) == learns


def _steps_asked(monkeypatch):
    """The parameters (their number) and the step's number of each call of the library."""
    asked = []
    monkeypatch.setattr(B, "load", lambda: type("Library", (), {"moe_adamw": staticmethod(lambda *args: asked.append((args[1], args[12])) or 0), "moe_adamw_check": lambda *_: 0})())
    return asked


def test_a_parameters_steps_are_its_own(on_host, monkeypatch):
    asked = _steps_asked(monkeypatch)
    early, late, never = (torch.zeros(4, requires_grad=True) for _ in range(3))
    one = AdamW([early, late, never])
    one.step()                                                              # (no gradient anywhere: no step)
    assert asked == [] and one.steps == 0
    early.grad = torch.zeros(4)
    one.step(), one.step()
    late.grad = torch.zeros(4)
    one.step()
    early.grad = None
    one.step()
    assert asked == [(1, 1), (1, 2), (1, 3), (1, 1), (1, 2)] and one.counts == [3, 2, 0] and one.steps == 3
    other = AdamW([torch.zeros(4) for _ in range(3)])
    other.load_state_dict(one.state_dict())
    one.step()
    assert other.counts == [3, 2, 0]
    other.load_state_dict(dict(one.state_dict(), steps=7))                  # a state with one count for all
    assert other.counts == [7, 7, 7]
    with pytest.raises(B.MoeError):
        other.load_state_dict(dict(one.state_dict(), steps=[1, 2]))
    assert other.counts == [7, 7, 7]


def test_a_refused_step_changes_nothing(lib, on_host, monkeypatch):
    """Whatever refuses it, in the first group of parameters or the last: no call is made, no step counted, no version moved; the next step is the first."""
    asked = []
    library = type("Library", (), {"moe_adamw": staticmethod(lambda *args: asked.append(args[12]) or lib.moe_adamw_check(*args[:-1])), "moe_adamw_check": lib.moe_adamw_check,
                                   "moe_last_error": lib.moe_last_error})
    monkeypatch.setattr(B, "load", lambda: library)
    for halves in (False, True):
        params = [torch.zeros(4, requires_grad=True)] + [torch.zeros(4, dtype=torch.float16, requires_grad=True)] * halves
        one = AdamW(params)

        def refused(match, grad_scale=1.0):
            before = one.counts, [p._version for p in params]
            with pytest.raises(B.MoeError, match=match):
                one.step(grad_scale)
            assert (asked == [] or not halves) and one.steps == 0 and before == (one.counts, [p._version for p in params])
            asked.clear()

        for p in params:
            p.grad = torch.zeros_like(p)
        for scale in (float("inf"), float("nan")):
            refused("finite", scale)
        one.eps = -1.0
        refused("eps")
        one.eps = 1e-8
        state = one.exp_avg_sq[-1]
        one.exp_avg_sq[-1] = torch.zeros(5)
        refused("moment")
        one.exp_avg_sq[-1] = torch.frombuffer(bytearray(20), dtype=torch.uint8)[1:17].view(torch.uint8)
        refused("moment")
        one.exp_avg_sq[-1] = state
        one.step()
        assert one.counts == [1] * len(params) and asked == [1] * len(params)
        asked.clear()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_others_write_into_a_parameter_goes_into_its_master(on_host, dtype):
    p = torch.tensor([1.0, 2.0, 3.0, float("nan")]).to(dtype).requires_grad_()
    p.grad = torch.zeros_like(p)
    one = AdamW([p])
    with torch.no_grad():
        one.masters[0][:2] += 2.0 ** -14                                    # (what 16 bits do not show)
        one.step()
        assert one.masters[0][:3].tolist() == [1.0 + 2.0 ** -14, 2.0 + 2.0 ** -14, 3.0]
        p[1] = -5.0
        p.clamp_(max=2.5)
        one.step()
    assert one.masters[0][:3].tolist() == [1.0 + 2.0 ** -14, -5.0, 2.5] and bool(one.masters[0][3].isnan())
    with torch.no_grad():                                                   # a state, and then the parameters that belong to it: the state's masters stay
        other = torch.zeros(4, dtype=dtype)
        two = AdamW([other])
        two.load_state_dict(one.state_dict())
        other.grad = torch.zeros_like(other)
        other.copy_(p)
        two.step()
    assert two.masters[0][:3].tolist() == one.masters[0][:3].tolist()


def test_gradients_that_begin_between_16_bytes_are_copied():
    from paper_2211_10017_amd.exchange import whole
    room = torch.arange(200.0).half()
    at = next(i for i in range(8) if room[i:].data_ptr() % 16)
    part = room[at:at + 64].view(8, 8)
    assert part.is_contiguous() and whole(part).data_ptr() % 16 == 0 and torch.equal(whole(part), part)
    aligned = torch.zeros(8, 8)
    assert whole(aligned).data_ptr() == aligned.data_ptr() and whole(aligned.t()).is_contiguous()


def test_rows_of_adapters_are_counted_in_32_bits():
    """Above 2^30 rows a row's number and what is requested ahead of it could pass 2^31: refused, db alone among them, which needs no launch for the rows themselves."""
    def db(R):
        name, args = _calls(R, 1, 1, 64, 8, 16)[1]
        args[19] = PTR
        args[20] = args[22] = None                                          # no dx, no da
        return name, args
    assert [c.rc for c in record([db(2 ** 31 - 1), db(2 ** 30 + 1), _calls(2 ** 30 + 1, 1, 1, 64, 64, 16)[0]])] == [UNSUPPORTED] * 3
    got = record([db(2 ** 30)])[0]
    assert got.rc == OK and len(got.launches) == 2 and all(0 < l.grid[0] * l.block < 2 ** 32 for l in got.launches)


def test_which_order_an_index_stands_for():
    from paper_2211_10017_amd.adapters import AdapterIndex, LayerIndex
    assert AdapterIndex(1, 2, 3, 1).by_assignment and not AdapterIndex(1, 2, 3, 2).by_assignment
    assert not LayerIndex(1, 2, 3, 1).by_assignment and LayerIndex(1, 2, 3, 1) == (1, 2, 3, 1) and isinstance(LayerIndex(1, 2, 3, 1)._replace(k=2), LayerIndex)


def test_which_blocks_the_rows_go_through():
    """The sizes that the tests compare reach every block of adapter_kernel with eight wavefronts: <x, matrices, y, adds y, 8, sixteens of rows, sixteens of the rank>."""
    sizes = {(4700, 16): (2, 1), (4700, 24): (2, 2), (9001, 9): (3, 1), (9001, 32): (3, 2), (14999, 16): (5, 1), (14999, 20): (5, 2), (24000, 32): (5, 2), (17800, 5): (5, 1), (14000, 64): (2, 4),
             (9001, 64): (3, 4), (13500, 64): (4, 4), (14000, 100): (2, 8), (9900, 100): (3, 8)}
    calls = [c for R, rank in sizes for c in _calls(R, 1, 7, 72, 136, rank)]
    got = record(calls)
    for i, ((R, rank), (rows, ranks)) in enumerate(sizes.items()):
        for call, adds_y in zip(got[2 * i:2 * i + 2], ("true", "false")):
            assert call.rc == OK and call.launches[0].kernel == "adapter_kernel<0, 0, 0, %s, 8, %d, %d>" % (adds_y, rows, ranks), (R, rank, call.launches[0])


def test_a_state_that_was_not_copied_stays_whole(on_host, monkeypatch):
    """A state dict holds the optimiser's tensors as they are, and so it does the counts: loaded back after further steps it is the present state, not old counts beside new moments."""
    _steps_asked(monkeypatch)
    p = torch.zeros(4, requires_grad=True)
    p.grad = torch.zeros(4)
    one = AdamW([p])
    one.step()
    state = one.state_dict()
    one.step()
    assert state["steps"] == [2] and state["exp_avg"][0] is one.exp_avg[0]
    one.load_state_dict(state)
    assert one.counts == [2]
    one.step()
    assert state["steps"] == [3]


def test_tokens_and_rows_that_do_not_fit(on_host, monkeypatch):
    """permute_tokens and combine_tokens: the library knows neither how many rows there are nor how long the index is."""
    z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt)  # noqa: E731
    i32 = torch.int32
    permute_tokens(z(4, 64), z(4, 2, dt=i32), 8)
    for bad in ((z(3, 64), z(4, 2, dt=i32)), (z(5, 64), z(4, 2, dt=i32)), (z(64), z(4, 2, dt=i32)), (z(4, 64), z(4, dt=i32))):
        with pytest.raises(B.MoeError, match=r"\[T, k\]"):
            permute_tokens(*bad, 8)
    fine = dict(y_perm=z(8, 64), inv_perm=z(8, dt=i32), expert_scale=z(4, 2), active_rows=z(1, dt=i32))
    combine_tokens(**fine)
    combine_tokens(**dict(fine, y_perm=z(5, 64)))                           # (the active rows alone)
    combine_tokens(**dict(fine, y_perm=z(20, 64), active_rows=None))        # (some of a batch's tokens)
    with pytest.raises(B.MoeError, match="active_rows"):
        combine_tokens(**dict(fine, y_perm=z(7, 64), active_rows=None))
    for bad in (dict(y_perm=z(8 * 64)), dict(inv_perm=z(7, dt=i32)), dict(inv_perm=z(9, dt=i32)), dict(expert_scale=z(5, 2)), dict(expert_scale=z(8)), dict(active_rows=z(0, dt=i32))):
        with pytest.raises(B.MoeError, match=r"\[T \* k"):
            combine_tokens(**dict(fine, **bad))
    called = len(on_host)
    monkeypatch.setattr(B, "_raw_device", lambda: 1)
    for call in (lambda: combine_tokens(**fine), lambda: permute_tokens(z(4, 64), z(4, 2, dt=i32), 8)):
        with pytest.raises(B.MoeError, match="device"):
            call()
    assert len(on_host) == called


def test_an_index_is_made_where_the_call_runs(on_host, monkeypatch):
    adapters, idx = LowRankAdapters(2, 4, 64, 64, device="cpu"), torch.zeros(4, dtype=torch.int32)
    monkeypatch.setattr(B, "moe_permute_workspace_bytes", lambda *_: 16)
    assert adapters.index(idx).offsets.numel() == 3
    monkeypatch.setattr(B, "_raw_device", lambda: 1)
    with pytest.raises(B.MoeError, match="device"):
        adapters.index(idx)
    with pytest.raises(B.MoeError, match="device"):
        adapters.index(idx.long())


def test_the_number_of_steps_can_be_set(on_host, monkeypatch):
    asked = _steps_asked(monkeypatch)
    p = torch.zeros(4, requires_grad=True)
    p.grad = torch.zeros(4)
    one = AdamW([p])
    one.steps = 10                                                          # (a program that goes on with moments of its own)
    one.step()
    assert asked == [(1, 11)] and one.steps == 11
