"""Buffers of the caller's that do not fit the call are refused on the host, before their pointers go anywhere."""
import pytest
import torch

from paper_2211_10017_amd import binding as B


@pytest.mark.parametrize("bad", [dict(perm_src=15), dict(inv_perm=15), dict(offsets=8), dict(ws_dtype=torch.int32)])
def test_permute_index_refuses_buffers_that_do_not_fit(monkeypatch, bad):
    """8 tokens, two of 8 experts: 16 assignments and 9 offsets."""
    called = []

    class Library:
        moe_permute = staticmethod(lambda *args: called.append(args) or 0)

    monkeypatch.setattr(B, "load", lambda: Library)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    size = dict(perm_src=16, inv_perm=16, offsets=9, ws_dtype=torch.uint8)
    call = lambda s: B.moe_permute_index(torch.zeros((8, 2), dtype=torch.int32), 8, 64, torch.float16, *(torch.zeros(s[n], dtype=torch.int32) for n in  # noqa: E731
                                         ("perm_src", "inv_perm", "offsets")), torch.zeros(64, dtype=s["ws_dtype"]))
    call(size)
    call(dict(size, perm_src=20, inv_perm=17, offsets=12))                           # larger ones are taken
    assert len(called) == 2
    with pytest.raises(B.MoeError):
        call(dict(size, **bad))
    assert len(called) == 2


@pytest.mark.parametrize("finished", [torch.zeros(15, dtype=torch.uint8), torch.zeros(17, dtype=torch.uint8), torch.zeros(16, dtype=torch.bool), torch.zeros((16, 2), dtype=torch.uint8)[:, 0],
                                      torch.zeros(16, dtype=torch.int32)])
def test_layer_refuses_a_mask_that_does_not_fit(monkeypatch, finished):
    """The gate reads a byte of it per token."""
    from paper_2211_10017_amd import MoEMx4Layer
    layer = MoEMx4Layer(16, 64, 64, 8, 2, device="cpu")
    called = []

    class Library:
        moe_gate_topk = staticmethod(lambda *args: called.append(args) or 0)
        moe_permute = staticmethod(lambda *args: 0)

    monkeypatch.setattr(B, "load", lambda: Library)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    x = torch.zeros((16, 64), dtype=torch.float16)
    layer.route(x, torch.zeros(16, dtype=torch.uint8))
    layer.route(x)
    assert len(called) == 2
    with pytest.raises(B.MoeError, match="finished"):
        layer.route(x, finished)
    assert len(called) == 2
