"""What a layer is tuned with, run together: sorting and combining with gradients, adapters, AdamW, beside the layers; against torch's own differentiation of the formulas in 64 bits."""
import pytest
import torch

from paper_2211_10017_amd import (AdamW, LowRankAdapters, MoEExpertLayer, MoEMx4Layer, adapt, adapter_index, balance_loss, combine_tokens, permute_tokens)
from paper_2211_10017_amd import binding as B
from paper_2211_10017_amd.adapters import AdapterIndex
from paper_2211_10017_amd.mx4_router_tuning import tune
from tuning_ref import BF16, F16, F32, U, adapters_ref, generator, routing, sorted_index, within

pytestmark = pytest.mark.gpu


def r(gen, *s):
    return torch.randn(s, generator=gen, device="cuda")


@pytest.mark.parametrize("T,k,d,load", [(1, 1, 8, "even"), (65, 2, 72, "pruned"), (300, 2, 264, "even"), (40, 2, 64, "none"), (5000, 1, 64, "pruned")])
def test_there_and_back_with_gradients(T, k, d, load):
    """x sorted, multiplied row by row, and combined: gradients of x, of the factors and of the scales."""
    gen, E = generator(T), 8
    idx = routing(gen, T, k, E, load)
    x, w, scale, dout = r(gen, T, d), r(gen, T * k, d), torch.rand((T, k), generator=gen, device="cuda"), r(gen, T, d)
    ours = [t.clone().requires_grad_() for t in (x, w, scale)]
    x_perm, perm_src, inv, offsets = permute_tokens(ours[0], idx, E)
    out = combine_tokens(x_perm * ours[1], inv, ours[2], active_rows=offsets[E:])
    (out * dout).sum().backward()
    theirs = [t.double().requires_grad_() for t in (x, w, scale)]
    perm, inv64, off = sorted_index(idx, E)
    live = (torch.arange(T * k, device="cuda") < int(off[E]))[:, None]
    y = theirs[0][perm.long() // k] * theirs[1] * live
    want = (y[inv64.long()].view(T, k, d) * theirs[2][:, :, None]).sum(1)
    (want * dout.double()).sum().backward()
    assert torch.equal(inv, inv64) and torch.equal(perm_src, perm) and torch.equal(offsets, off)
    mag = (y[inv64.long()].view(T, k, d) * theirs[2][:, :, None]).abs().sum(1)
    within(out.detach(), want.detach(), 8 * U * mag.detach())
    # products of up to three factors and sums of k terms (d for the scales)
    dwmag = theirs[1].grad.abs()
    within(ours[1].grad, theirs[1].grad, 8 * U * dwmag)
    parts = (dout.double().repeat_interleave(k, 0) * (theirs[0][torch.arange(T, device="cuda").repeat_interleave(k)] * theirs[1].detach()[inv64.long()]).detach()).abs()
    within(ours[2].grad, theirs[2].grad, (d + 8) * U * parts.sum(1).view(T, k))
    dx = (dout.double().repeat_interleave(k, 0) * theirs[1].detach()[inv64.long()] * theirs[2].detach().view(-1, 1)).abs().view(T, k, d).sum(1)
    within(ours[0].grad, theirs[0].grad, 8 * U * dx)


@pytest.mark.parametrize("xt,yt", [(F16, F32), (BF16, BF16)])
@pytest.mark.parametrize("T,k,by", [(70, 1, True), (70, 1, False), (70, 2, False), (70, 2, True), (1100, 2, False), (1, 1, True)])
def test_adapters_with_gradients(T, k, by, xt, yt):
    gen, E, K, N, rank = generator(T + k), 5, 136, 72, 12
    idx = routing(gen, T, k, E, "pruned" if T > 1 else "even")
    perm, inv, offsets = sorted_index(idx, E)
    index = (adapter_index(idx.view(-1), E) if k == 1 else None)
    if index is None:
        from paper_2211_10017_amd import AdapterIndex
        index = AdapterIndex(perm, inv, offsets, k)
    assert torch.equal(index.perm_src, perm) and torch.equal(index.inv_perm, inv) and torch.equal(index.offsets, offsets)
    x, a, b = r(gen, T, K).to(xt), (r(gen, E, rank, K) * K ** -0.5).to(xt), r(gen, E, rank, N).to(xt)
    y, scale, dout = r(gen, T * k, N).to(yt), torch.rand(E, generator=gen, device="cuda"), r(gen, T * k, N).to(yt)
    ours = [t.clone().requires_grad_() for t in (x, y, a, b)]
    out = adapt(*ours, index, scale, by_assignment=by)
    want = adapters_ref(x, a, b, offsets, perm, k, scale, by, y, dout)
    (out * dout).sum().backward()
    within(out.detach(), want["out"], want["out_mag"] + 2.0 ** -23 * (want["out"].abs() + y.double().abs()))
    assert torch.equal(ours[1].grad, dout)
    within(ours[2].grad, want["da"], want["da_mag"] + 2.0 ** -23 * want["da"].abs())
    within(ours[3].grad, want["db"], want["db_mag"] + 2.0 ** -23 * want["db"].abs())
    rows = torch.arange(T * k, device="cuda") if by else inv.long()
    dx, mag = (want[n][rows].view(T, k, K) for n in ("dx", "dx_mag"))
    # each row is rounded to x's type before the token's are added
    rounding = torch.finfo(xt).eps / 2 * dx.abs().sum(1) + 2.0 ** -25
    within(ours[0].grad, dx.sum(1), mag.sum(1) + rounding)
    alone = adapt(x, None, a, b, index, scale, by_assignment=by, y_dtype=F32)
    assert alone.dtype == F32 and alone.shape == (T * k, N)


def test_what_changes_in_between_is_seen_or_does_not_matter():
    """The index may be written again before the backward pass; the rows may not: a layer's next call, an optimiser's step and torch's own writes raise."""
    gen, T, k, d, F, E = generator(1), 64, 2, 128, 128, 8
    layer = MoEMx4Layer(T, d, F, E, k)
    for e in range(E):
        layer.load_expert(1, e, r(gen, d, F) * 0.1)
        layer.load_expert(2, e, r(gen, F, d) * 0.1)
    layer.wg.copy_(r(gen, d, E) * 0.1)
    x, other = r(gen, T, d).half(), r(gen, T, d).half()
    adapters = LowRankAdapters(E, 4, d, d, generator=gen)
    adapters.b.normal_(generator=gen)
    adapters.requires_grad_()

    def forward():
        layer.route(x)
        layer.experts(x)
        scale = layer.expert_scale.clone().requires_grad_()
        y = adapters(x, layer.y_perm.clone(), layer.index())
        return scale, combine_tokens(y, layer.inv_perm, scale, active_rows=layer.expert_offsets[E:])

    scale, out = forward()
    out.square().sum().backward()
    want = [t.grad.clone() for t in (scale, adapters.a, adapters.b)]
    adapters.a.grad = adapters.b.grad = None
    scale, out = forward()
    layer.route(other)                                              # the same buffers hold another index now
    layer.experts(other)
    out.square().sum().backward()
    assert all(torch.equal(t.grad, w) for t, w in zip((scale, adapters.a, adapters.b), want))
    layer.route(x)
    layer.experts(x)
    scale = layer.expert_scale.clone().requires_grad_()
    out = combine_tokens(layer.y_perm, layer.inv_perm, scale, active_rows=layer.expert_offsets[E:])
    layer.experts(x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    scale, out = forward()
    AdamW(adapters.parameters()).step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    rows = x.float().repeat(2, 1).requires_grad_()
    scale, out = forward()
    sorted_rows = permute_tokens(rows, torch.zeros((2 * T, 1), dtype=torch.int32, device="cuda"), E)[0]
    for out, leaves in ((out, [scale]), (out, adapters.parameters()), (sorted_rows, [rows])):
        grads = torch.autograd.grad(out.square().sum(), leaves, create_graph=True, retain_graph=True)
        with pytest.raises(B.MoeError, match="second derivative"):
            sum(g.square().sum() for g in grads).backward(retain_graph=True)


def test_a_tuning_step_against_64_bits():
    """Balance loss, scales, adapters and combine in one graph over a layer's own rows, and what AdamW makes of the gradients."""
    gen, T, k, d, F, E, rank, coef = generator(3), 96, 2, 128, 192, 8, 6, 0.05
    layer = MoEMx4Layer(T, d, F, E, k)
    for e in range(E):
        layer.load_expert(1, e, r(gen, d, F) * 0.1)
        layer.load_expert(2, e, r(gen, F, d) * 0.1)
    layer.wg.copy_(r(gen, d, E) * 0.1)
    x, target = r(gen, T, d).half(), r(gen, T, d)
    finished = (torch.rand(T, generator=gen, device="cuda") < 0.2).to(torch.uint8)
    adapters = LowRankAdapters(E, rank, d, d, alpha=12, generator=gen)
    adapters.b.normal_(generator=gen).mul_(0.1)
    adapters.requires_grad_()
    wg = layer.wg.float().requires_grad_()
    layer.route(x, finished)
    layer.experts(x)
    active = layer.expert_offsets[E:]
    scale, loss, _, _ = balance_loss(x.float() @ wg, layer.expert_idx, coef)
    out = combine_tokens(adapters(x, layer.y_perm, layer.index()), layer.inv_perm, scale, active_rows=active)
    total = (out - target).square().mean() + loss
    total.backward()
    # the same in 64 bits, differentiated by torch
    wg64, a64, b64 = (t.detach().double().requires_grad_() for t in (wg, adapters.a, adapters.b))
    p = torch.softmax(x.double() @ wg64, 1)
    idx = layer.expert_idx.long()
    live = (idx < E).all(1)
    chosen = p.gather(1, idx.clamp(max=E - 1)) * live[:, None]
    s64 = torch.where(live[:, None], chosen / chosen.sum(1, keepdim=True).clamp(min=1e-300), 0.0)
    counts = torch.bincount(idx[live].flatten(), minlength=E).double()
    loss64 = coef * E * (counts / counts.sum() * p[live].mean(0)).sum()
    y = layer.y_perm.double().index_select(0, layer.inv_perm.long().view(-1))
    u = torch.einsum("td,tkjd->tkj", x.double(), a64[idx.clamp(max=E - 1)])
    delta = torch.einsum("tkj,tkjn->tkn", u, b64[idx.clamp(max=E - 1)]) * 2.0
    y_new = y.view(T, k, d) + delta
    y_new = y_new + (y_new.half().double() - y_new).detach()                 # y is stored in fp16: the rounded value, the gradient of the sum
    y_new = torch.where(live[:, None, None], y_new, 0.0)
    out64 = (s64[:, :, None] * y_new).sum(1)
    total64 = (out64 - target.double()).square().mean() + loss64
    total64.backward()
    assert abs(float(total.detach() - total64.detach())) <= 1e-3 * float(total64.detach())              # (fp16 rows: half a step is 2^-11 of y, and y is a part of the error)
    for got, want in ((wg.grad, wg64.grad), (adapters.a.grad, a64.grad), (adapters.b.grad, b64.grad)):
        # gradients pass through rows and gradients of rows in fp16 (2^-11 each, four on the way), and are rounded to their type: in the mean over an array far below 2^-8
        assert float((got.double() - want).norm() / want.norm()) <= 2.0 ** -8
    params = [wg] + adapters.parameters()
    before, grads = [t.detach().double().clone() for t in params], [t.grad.double().clone() for t in params]
    AdamW(params, lr=0.1, weight_decay=0.0).step()
    for t, old, g in zip(params, before, grads):
        # the first step's moments are (1 - b) g: the step is lr g / (|g| + eps)
        want = old - 0.1 * g / (g.abs() + 1e-8)
        within(t.detach(), want, 32 * U * (0.1 + old.abs()))


def test_adapters_in_the_layers():
    gen, T, k, d, F, E = generator(4), 80, 2, 128, 256, 8
    layer = MoEMx4Layer(T, d, F, E, k, act_dtype=BF16)
    for e in range(E):
        layer.load_expert(1, e, r(gen, d, F) * 0.1)
        layer.load_expert(2, e, r(gen, F, d) * 0.1)
    layer.wg.copy_(r(gen, d, E) * 0.1)
    x = r(gen, T, d).to(BF16)
    finished = (torch.rand(T, generator=gen, device="cuda") < 0.3).to(torch.uint8)
    base = layer.forward(x, finished).clone()
    y = layer.y_perm.clone()
    layer.adapters = LowRankAdapters(E, 8, d, d, dtype=BF16, generator=gen)
    assert torch.equal(layer.forward(x, finished), base)                    # an adapter begins by changing nothing
    layer.adapters.b.normal_(generator=gen)
    out = layer.forward(x, finished)
    n = int(layer.expert_offsets[E])
    want = adapters_ref(x, layer.adapters.a, layer.adapters.b, layer.expert_offsets, layer.perm_src, k, layer.adapters.scale, False, torch.where((torch.arange(T * k, device="cuda") < n)[:, None], y, 0.0))
    within(layer.y_perm[:n], want["out"][:n], (want["out_mag"] + 2.0 ** -23 * (want["out"].abs() + y.double().abs().nan_to_num()))[:n])
    again = B.moe_combine(layer.y_perm, layer.inv_perm, layer.expert_scale, T, k, active_rows=layer.expert_offsets[E:])
    assert torch.equal(out, again) and bool((out[finished.bool()] == 0).all())
    # requests' adapters beside a layer of int4 experts, in its own output
    int4 = MoEExpertLayer(T, d, F, E, k, 4, act_dtype=BF16)
    for e in range(E):
        int4.load_expert(1, e, r(gen, d, F) * 0.1)
        int4.load_expert(2, e, r(gen, F, d) * 0.1)
    int4.wg.copy_(layer.wg)
    requests = LowRankAdapters(3, 16, d, d, dtype=BF16, generator=gen)
    requests.b.normal_(generator=gen)
    idx = torch.randint(0, 4, (T,), generator=gen, device="cuda").int()      # 3: none
    index = requests.index(idx)
    y0 = int4.forward(x).clone()
    got = requests.add(x, int4.forward(x), index)
    assert got is int4.out
    want = adapters_ref(x, requests.a, requests.b, index.offsets, index.perm_src, 1, requests.scale, True, y0)
    within(got, want["out"], want["out_mag"] + 2.0 ** -23 * (want["out"].abs() + y0.double().abs()))
    assert torch.equal(got[idx == 3], y0[idx == 3])


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_a_program(bits):
    """Parameters of several types, one without a gradient, a state that is saved and loaded."""
    gen = generator(bits)
    make = lambda: [t.requires_grad_() for t in (r(generator(1), 300), r(generator(2), 40, 16).half(), r(generator(3), 7), r(generator(4), 64, 8).to(BF16), r(generator(5), 33))]  # noqa: E731
    a, b = make(), make()
    kw = dict(lr=0.01, betas=(0.8, 0.95), weight_decay=0.1, bits=bits)
    one, two = AdamW(a, **kw), AdamW(b, **kw)
    ref = [t.detach().double() for t in a]
    m, v = [torch.zeros_like(t) for t in ref], [torch.zeros_like(t) for t in ref]
    for t in range(1, 5):
        for i, (p, q) in enumerate(zip(a, b)):
            if i == 2:
                continue
            p.grad = r(gen, *p.shape).to(p.dtype)
            q.grad = p.grad.clone()
            g = p.grad.double() * 0.5
            m[i], v[i] = 0.8 * m[i] + 0.2 * g, 0.95 * v[i] + 0.05 * g * g
            ref[i] = ref[i] * (1 - 0.01 * 0.1) - 0.01 / (1 - 0.8 ** t) * m[i] / ((v[i] / (1 - 0.95 ** t)).sqrt() + 1e-8)
        one.step(grad_scale=0.5)
        two.step(grad_scale=0.5)
        if t == 2:                                                          # a program that stops here and goes on with what it saved
            saved, values = two.state_dict(), [q.detach().clone() for q in b]
            b = [q.requires_grad_() for q in values]
            fresh = AdamW(b, **kw)
            fresh.load_state_dict(saved)
            two = fresh
        if bits == 32:
            for p, w in zip(a, ref):
                # four steps of fp32 arithmetic, 16 roundings of the value and of a step of 0.01 each; the first is at most twice the rate
                within(p.detach(), w, 4 * 16 * U * (w.abs() + 0.02))
    assert all(torch.equal(p, q) for p, q in zip(a, b)) and torch.equal(a[2].detach(), r(generator(3), 7)) and one.steps == 4
    one.zero_grad(set_to_none=False)
    assert all(bool((p.grad == 0).all()) for p in a if p.grad is not None)
    one.zero_grad()
    assert all(p.grad is None for p in a)


def test_a_captured_step_replays():
    """Forward, gradients and AdamW as one graph, with the step's number on the device: several replays with the program's own work between them, against the same calls one by one."""
    gen, T, k, d, E, rank = generator(7), 64, 2, 128, 4, 8
    idx = routing(gen, T, k, E, "pruned")
    perm, inv, offsets = sorted_index(idx, E)
    from paper_2211_10017_amd import AdapterIndex
    index = AdapterIndex(perm, inv, offsets, k)
    x, target = torch.empty((T, d), dtype=F16, device="cuda"), r(gen, T, d)
    y, scale = r(gen, T * k, d), torch.rand((T, k), generator=gen, device="cuda").requires_grad_()

    def program():
        a, b = ((r(generator(8 + i), E, rank, d) * 0.1).half().requires_grad_() for i in range(2))
        masters, grads = [t.detach().float() for t in (a, b)], [torch.zeros_like(t, requires_grad=False) for t in (a, b)]
        m, v = ([torch.zeros_like(t) for t in masters] for _ in range(2))
        step = torch.zeros(1, dtype=torch.int32, device="cuda")

        def run():
            out = combine_tokens(adapt(x, y, a, b, index), inv, scale, active_rows=offsets[E:])
            got = torch.autograd.grad((out - target).square().mean(), [a, b])
            for g, n in zip(grads, got):
                g.copy_(n)
            step.add_(1)
            B.moe_adamw(masters, grads, m, v, step, lr=0.01, copies=[a.detach(), b.detach()])
            return out.detach()

        return run, (masters, m, v, grads, [a.detach(), b.detach()])

    x.normal_(generator=gen)
    warm, _ = program()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            warm()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    captured, state = program()
    eager, want = program()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = captured()
    for rep in range(5):
        x.normal_(generator=gen)
        torch.cuda.synchronize()
        graph.replay()
        expected = eager()
        torch.cuda.synchronize()
        assert torch.equal(out, expected), rep
        for s, w in zip(state, want):
            assert all(torch.equal(p, q) for p, q in zip(s, w)), rep


@pytest.mark.parametrize("optimizer", ["sgd", "adamw", "adamw8"])
def test_the_tuning_command_with_adapters_runs(optimizer):
    lines = []
    first, last, losses = tune(steps=3, T=64, d=128, F=128, E=8, adapter_rank=4, optimizer=optimizer, report=lines.append)
    assert len(losses) == 3 and all(0 < v < 100 for v in losses + [first, last]) and len(lines) == 2


@pytest.mark.parametrize("k,by_assignment", [(1, True), (1, False), (2, False)])
def test_no_tokens_at_all(k, by_assignment):
    """An empty batch through the functions with gradients: empty rows, gradients of 0 for the matrices."""
    a = LowRankAdapters(4, 8, 64, 72).requires_grad_()
    x = torch.zeros((0, 64), dtype=F16, device="cuda", requires_grad=True)
    rows = torch.empty(0, dtype=torch.int32, device="cuda")
    out = a(x, None, AdapterIndex(rows, rows, torch.zeros(5, dtype=torch.int32, device="cuda"), k), by_assignment=by_assignment)
    out.float().sum().backward()
    torch.cuda.synchronize()
    assert out.shape == (0, 72) and x.grad.shape == (0, 64) and bool((a.a.grad == 0).all()) and bool((a.b.grad == 0).all())


def test_adding_in_place_counts_as_a_change():
    """Autograd must not take y's rows for those that it kept."""
    gen, T = generator(7), 40
    requests = LowRankAdapters(4, 8, 64, 64)
    requests.b.normal_(generator=gen)
    x, w = r(gen, T, 64).half(), r(gen, T, 64).half().requires_grad_()
    index = requests.index(torch.zeros(T, dtype=torch.int32, device="cuda"))
    y = w * 2.0
    kept = y.square()
    requests.add(x, y.detach(), index)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.float().sum().backward()
    with torch.inference_mode():
        z = torch.zeros((T, 64), dtype=F16, device="cuda")
        assert requests.add(x, z, index) is z and bool((z != 0).any())
    with pytest.raises(B.MoeError, match="out is x"):
        requests.add(x, x, index)
