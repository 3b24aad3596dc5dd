"""What the 4-bit operators and the balance loss refuse, on the host, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2211_10017_amd import binding as B

P = ctypes.c_void_p(0x1000)          # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1008)
ARG, UNSUPPORTED, WORKSPACE = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    return B.load()


def test_quantisers_refuse(lib):
    rows, experts, back = lib.moe_mx4_quantize_rows, lib.moe_mx4_quantize_experts, lib.moe_mx4_dequantize
    assert rows(P, 0, 4, 96, 96, P, P, None) == ARG and b"multiple of 64" in lib.moe_last_error()
    assert rows(P, 0, -1, 64, 64, P, P, None) == ARG and rows(P, 0, 4, 64, 32, P, P, None) == ARG and rows(P, 0, 4, 64, 68, P, P, None) == ARG
    assert rows(P, 3, 4, 64, 64, P, P, None) == UNSUPPORTED and rows(None, 0, 4, 64, 64, P, P, None) == ARG and rows(ODD, 0, 4, 64, 64, P, P, None) == ARG
    assert rows(None, 0, 0, 64, 64, None, None, None) == 0
    assert experts(P, 1, 64, 40, P, P, None) == ARG and experts(P, 1, 32, 64, P, P, None) == ARG and experts(P, 1, 64, 64, P, None, None) == ARG
    assert back(P, P, 1, 4, 64, P, 7, None) == UNSUPPORTED and back(P, P, 1, 4, 100, P, 0, None) == ARG and back(P, ODD, 1, 4, 64, P, 0, None) == ARG


def test_products_refuse(lib):
    gemm = lambda a=P, rows=8, src=P, k=1, off=P, R=8, E=2, most=0, K=64, N=32, w=P, bias=None, act=-1, y=P, dt=0: lib.moe_grouped_gemm_mx4(  # noqa: E731
        a, P, rows, src, k, off, R, E, most, K, N, w, P, bias, act, y, dt, None)
    for bad in (dict(K=32), dict(K=96), dict(N=16), dict(N=48), dict(R=-1), dict(k=0), dict(src=None, rows=7), dict(a=None), dict(y=None), dict(off=None), dict(w=ODD), dict(bias=ODD),
                dict(most=-1)):
        assert gemm(**bad) == ARG, bad
    for bad in (dict(dt=3), dict(act=2), dict(act=-2), dict(E=4097), dict(K=(1 << 24) + 64), dict(N=(1 << 24) + 32)):
        assert gemm(**bad) == UNSUPPORTED, bad
    assert gemm(R=0) == 0 and gemm(E=0) == 0
    ffn = lambda x=P, dt=0, T=8, R=8, d=64, F=64, act=0, y=P, ydt=0, ws=P, size=1 << 30, b1=None: lib.moe_grouped_ffn_mx4(  # noqa: E731
        x, dt, T, P, 1, P, R, 2, 0, d, F, act, P, P, b1, P, P, None, y, ydt, ws, size, None)
    for bad in (dict(d=96), dict(F=96), dict(x=None), dict(y=ODD), dict(b1=ODD), dict(T=-1), dict(ws=ODD)):
        assert ffn(**bad) == ARG, bad
    for bad in (dict(dt=4), dict(ydt=-1), dict(act=-1), dict(act=3)):
        assert ffn(**bad) == UNSUPPORTED, bad
    need = lib.moe_grouped_ffn_mx4_workspace_bytes(8, 8, 64, 64)
    assert need >= 2 * (8 * 32 + 8 * 4) and ffn(size=need - 1) == WORKSPACE and b"workspace" in lib.moe_last_error()
    assert ffn(ws=None) == WORKSPACE and ffn(R=0) == 0
    assert lib.moe_grouped_ffn_mx4_workspace_bytes(1 << 20, 1 << 21, 4096, 16384) > 1 << 34


def test_balance_loss_refuses(lib):
    fwd = lambda z=P, dt=2, idx=P, T=8, E=4, k=2, loss=P, scale=P, ws=P, size=1 << 30: lib.moe_balance_loss(  # noqa: E731
        z, dt, idx, T, E, k, 1, 0.01, loss, P, P, scale, P, ws, size, None)
    for bad in (dict(z=None), dict(z=ODD), dict(idx=None), dict(T=-1), dict(k=0), dict(k=5), dict(E=0), dict(loss=None), dict(scale=None), dict(ws=ODD)):
        assert fwd(**bad) == ARG, bad
    for bad in (dict(dt=3), dict(E=1025), dict(E=64, k=9)):
        assert fwd(**bad) == UNSUPPORTED, bad
    need = lib.moe_balance_loss_workspace_bytes(9000, 4)
    assert need > 0 and fwd(T=9000, size=need - 1) == WORKSPACE and fwd(T=9000, ws=None) == WORKSPACE and lib.moe_balance_loss_workspace_bytes(8, 4) == 0
    back = lambda w=P, out=P, T=8, E=4, dt=2: lib.moe_balance_loss_backward(P, dt, P, T, E, 2, 1, w, None, None, out, None)  # noqa: E731
    assert back(w=None) == ARG and back(out=ODD) == ARG and back(E=2000) == UNSUPPORTED and back(dt=-1) == UNSUPPORTED and back(T=0) == 0


def test_the_binding_refuses_tensors_that_do_not_fit():
    u8, f = (lambda *s: torch.zeros(s, dtype=torch.uint8)), torch.zeros
    with pytest.raises(B.MoeError, match="CUDA"):
        B.moe_mx4_quantize_rows(f(4, 64))
    with pytest.raises(B.MoeError, match="codes must be"):
        B.moe_mx4_dequantize(u8(4, 48), u8(1, 4, 4))
    with pytest.raises(B.MoeError, match="scales must be"):
        B.moe_mx4_dequantize(u8(4, 128), u8(1, 4, 4))
    off = torch.zeros(3, dtype=torch.int32)
    w, s = u8(2, 64, 32), u8(2, 1, 64, 4)
    with pytest.raises(B.MoeError, match="E \\+ 1 offsets"):
        B.moe_grouped_gemm_mx4(u8(4, 32), u8(1, 4, 4), torch.zeros(4, dtype=torch.int32), w, s)
    with pytest.raises(B.MoeError, match="weights' K"):
        B.moe_grouped_gemm_mx4(u8(4, 64), u8(1, 4, 4), off, w, s)
    with pytest.raises(B.MoeError, match="y must be"):
        B.moe_grouped_gemm_mx4(u8(4, 32), u8(1, 4, 4), off, w, s, y=f(4, 32))
    with pytest.raises(B.MoeError, match="w1 must be"):
        B.moe_grouped_ffn_mx4(f(4, 128), off, w, s, w, s)
    with pytest.raises(B.MoeError, match="expert_idx"):
        B.moe_balance_loss(f(4, 8), torch.zeros((3, 2), dtype=torch.int32))
    with pytest.raises(B.MoeError, match="weight must be"):
        B.moe_balance_loss_backward(f(4, 8), torch.zeros((4, 2), dtype=torch.int32), f(7))
