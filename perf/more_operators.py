"""What a layer of quantised experts is tuned and adapted with, for timing: the gradient of sorting tokens by expert and back, low-rank adapters of
many requests (or experts) beside a shared projection with their gradient, and an AdamW step over many tensors with states in 32 or 8 bits.
`run` calls them as users do, or, with `own` false, computes them in elementary torch operations.

The sizes are those of this repository's configurations, tests, tuning command and benchmark (d_model 256 to 4096, 8 to 128 experts, 1 to 16384
tokens) and generic ones beside them."""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4}


def _named(name, case, kw):
    case.update(kw)
    return dict(name=name, **case) if name else case


def _exchange(name=None, **kw):
    return _named(name, dict(op="exchange", T=512, k=2, E=16, d=256, y="f16", out="f32", load="even", finished=0.0), kw)


def _adapt(name=None, **kw):
    return _named(name, dict(op="adapt", T=64, k=1, E=32, K=1024, N=1024, rank=16, x="f16", y="f16", load="even", finished=0.0), kw)


def _gradient(name=None, **kw):
    return _named(name, dict(op="gradient", T=512, k=2, E=16, K=256, N=256, rank=8, x="f16", y="f16", grad="f16", load="even", finished=0.0), kw)


def _adamw(name=None, **kw):
    return _named(name, dict(op="adamw", tensors=2, n=32768, odd=False, bits=32, g="f32", copy=False), kw)


def listed():
    return [
        # the tuning command's layer: 512 tokens, two of 16 experts, gradient of the un-permute and of the permute
        _exchange("exchange_512"),
        # a ragged bf16 batch, y in fp32 as the layer keeps it, a quarter of the sentences ended, some experts busier than others
        _exchange("exchange_997_bf16", T=997, d=704, y="f32", out="bf16", load="uneven", finished=0.25),
        # the largest batch of the large layer
        _exchange("exchange_16384", T=16384, E=64, d=4096, out="f16"),
        # one request, one decoder step, its adapter one of eight beside a projection of d_model 1024
        _adapt("adapt_1", T=1, E=8),
        # a decoder batch of 64 requests with 32 adapters, a quarter of them without one, beside a projection of 1024 to 4096
        _adapt("adapt_64_bf16", N=4096, x="bf16", y="bf16", finished=0.25),
        # the largest: a prompt batch of requests, some adapters used more than others
        _adapt("adapt_16384_bf16", T=16384, K=4096, N=4096, rank=32, x="bf16", y="bf16", load="uneven"),
        # adapters of experts in the tuning command's layer: gradient of rows and of both matrices
        _gradient("gradient_512"),
        # a ragged bf16 batch with y in fp32 and an odd rank, pruned rows, gradients kept in fp32
        _gradient("gradient_997_bf16", T=997, K=704, N=2880, rank=12, x="bf16", y="f32", grad="f32", load="uneven", finished=0.25),
        # adapters of the large layer's experts
        _gradient("gradient_8192_bf16", T=8192, E=64, K=4096, N=4096, rank=16, x="bf16", y="bf16", grad="bf16"),
        # a router's weight and bias: launches and latency
        _adamw("adamw_router", odd=True),
        # adapters of 24 layers of the paper's model, both matrices: fp32 masters with 16-bit copies, 16-bit gradients
        _adamw("adamw_48", tensors=48, n=32 * 16 * 1024, g="bf16", copy=True),
        # adapters of the large layer's experts in 16 layers, states in 8 bits
        _adamw("adamw_32_8bit", tensors=32, n=64 * 16 * 4096, bits=8, g="bf16", copy=True),
    ]


_MAX_ROWS_BYTES = 16384 * 4096          # values of a tensor of rows in the largest listed cases
_MAX_PARAMETERS = 32 * 64 * 16 * 4096


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["exchange", "adapt", "adapt", "gradient", "gradient", "adamw"])
    load = rng.choice(["even", "even", "uneven"])
    k, E = rng.choice([1, 2]), rng.choice([2, 8, 16, 32, 61, 64, 128])
    x = rng.choice(["f16", "bf16"])
    if op == "adamw":
        tensors = _log_int(rng, 1, 100)
        return _adamw(tensors=tensors, n=_log_int(rng, 32, _MAX_PARAMETERS // tensors // 2), odd=rng.random() < 0.5, bits=rng.choice([32, 8]),
                      g=rng.choice(["f32", "f16", "bf16"]), copy=rng.random() < 0.5)
    if op == "exchange":
        d = 8 * _log_int(rng, 8, 512)
        T = _log_int(rng, 1, min(16384, _MAX_ROWS_BYTES // d))
        return _exchange(T=T, k=k, E=E, d=d, y=rng.choice(["f16", "bf16", "f32"]), out=rng.choice(["f16", "bf16", "f32"]), load=load,
                         finished=rng.choice([0.0, rng.uniform(0.1, 0.6)]) if T > 8 else 0.0)
    while True:
        K, N, rank = 8 * _log_int(rng, 8, 512), 8 * _log_int(rng, 8, 512), _log_int(rng, 1, 128)
        T = _log_int(rng, 1, 256) if op == "adapt" and rng.random() < 0.5 else _log_int(rng, 16, 16384)
        if T * k * max(K, N) <= _MAX_ROWS_BYTES // 2 and T * k * rank <= 16384 * 16:
            break
    y = rng.choice([x, x, "f32"])
    more = dict(T=T, k=k, E=E, K=K, N=N, rank=rank, x=x, y=y, load=load, finished=rng.choice([0.0, rng.uniform(0.1, 0.6)]) if T > 8 else 0.0)
    return _adapt(**more) if op == "adapt" else _gradient(grad=rng.choice([x, "f32"]), **more)


# ---- inputs -----------------------------------------------------------------------------------------------------------------------

def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _activations(gen, T, d):
    """Rows as layers see them: normally distributed, with channels of unlike size."""
    return _randn(gen, T, d) * torch.exp(0.5 * _randn(gen, d))


def _routing(gen, case):
    """Sorted index of a batch: expert (or adapter) of each assignment, perm_src, inv_perm, offsets and the most rows that an expert has."""
    T, k, E = case["T"], case["k"], case["E"]
    logits = _randn(gen, T, E) * 0.64
    if case["load"] == "uneven":
        logits = logits + (torch.rand(E, generator=gen, device="cuda") - 0.5) * 0.36
    idx = logits.topk(k, dim=1).indices
    if case["finished"]:
        idx[torch.randperm(T, generator=gen, device="cuda")[:max(1, round(case["finished"] * T))]] = E
    flat = idx.flatten()
    perm = torch.sort(flat, stable=True).indices
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(T * k, device="cuda")
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    return perm.to(torch.int32), inv.to(torch.int32), offsets, max(1, int(counts.max()))


def _starts(case):
    """Where each tensor of an AdamW case begins in the buffers, and its size: starts are multiples of 32."""
    n = case["n"]
    sizes = [max(1, n - (i * 7 + 1) % 31) if case["odd"] else n for i in range(case["tensors"])]
    room = (n + 31) // 32 * 32
    return [i * room for i in range(case["tensors"])], sizes, room * case["tensors"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op == "adamw":
        starts, sizes, total = _starts(case)
        real = torch.zeros(total, device="cuda")
        for a, n in zip(starts, sizes):
            real[a:a + n] = 1.0
        s["p"] = _randn(gen, total) * 0.02 * real
        g = _randn(gen, total) * torch.exp(_randn(gen, total)) * 1e-3 * real        # gradients of unlike size
        s["g"] = g.to(_DT[case["g"]])
        s["m"] = (0.3 * g + 1e-4 * _randn(gen, total)) * real
        s["v"] = (g * g * (0.5 + torch.rand(total, generator=gen, device="cuda")) + 1e-8) * real
        if case["bits"] == 8:
            s["m"], s["v"] = _hold(s["m"], False), _hold(torch.sqrt(s["v"]), True)
        s["copy"] = s["p"].to(torch.bfloat16) if case["copy"] else None
        cut = lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        held = lambda h: [(h[0][a:a + n], h[1][a // 32:(a + n + 31) // 32]) for a, n in zip(starts, sizes)]  # noqa: E731
        states = held if case["bits"] == 8 else cut
        s["tensors"] = dict(p=cut(s["p"]), g=cut(s["g"]), m=states(s["m"]), v=states(s["v"]), copy=cut(s["copy"]) if case["copy"] else None)
        s["step"] = 100
        return s
    T, k, E = case["T"], case["k"], case["E"]
    R = T * k
    s["perm_src"], s["inv_perm"], s["offsets"], s["cap"] = _routing(gen, case)
    if op == "exchange":
        d = case["d"]
        s["dout"] = (_randn(gen, T, d) * 1e-3).to(_DT[case["out"]])
        s["y"] = _activations(gen, R, d).to(_DT[case["y"]])
        s["scale"] = torch.rand((T, k), generator=gen, device="cuda") * 0.5 + 0.25
        s["dx_perm"] = (_randn(gen, R, d) * 1e-3).to(_DT["f16" if case["y"] == "f16" else "bf16"])
        return s
    K, N, rank = case["K"], case["N"], case["rank"]
    s["x"] = _activations(gen, T, K).to(_DT[case["x"]])
    s["a"] = (_randn(gen, E, rank, K) * K ** -0.5).to(_DT[case["x"]])
    s["b"] = (_randn(gen, E, rank, N) * 0.05).to(_DT[case["x"]])
    s["adapter_scale"] = torch.rand(E, generator=gen, device="cuda") + 0.5
    # one row per request (k = 1): y in the requests' order; experts' adapters: y as the FFN leaves it, sorted
    s["y"] = _randn(gen, R, N).to(_DT[case["y"]])
    if op == "gradient":
        s["dy"] = s.pop("y").mul_(1e-2)
        s["v"] = _grouped(s["x"].float()[s["perm_src"].long() // k], s["a"].float(), s["offsets"], s["cap"])
    return s


# ---- the plain form: elementary operations in 32 bits -----------------------------------------------------------------------------

def _pow2(e):
    """2^e in fp32, for whole -127 <= e <= 127, put together from its bits (2^-127 is a subnormal number)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _hold(v, root):
    """v [n] in 8 bits: e4m3 numbers in units of a power of two for each 32 values, that power's exponent + 127."""
    b = v.view(-1, 32)
    e = ((b.abs().amax(1, keepdim=True).view(torch.int32) >> 23) - 134).clamp(-127, 127)
    q = (b * _pow2(-e)).to(torch.float8_e4m3fn).float()
    q = torch.where((q == 0) & (b > 0), 2.0 ** -9, q) if root else q                  # the root of a second moment stays above 0
    return q.to(torch.float8_e4m3fn).view(torch.uint8).view(-1), (e + 127).to(torch.uint8).view(-1)


def _held(state):
    codes, scales = state
    return (codes.view(torch.float8_e4m3fn).float().view(-1, 32) * _pow2(scales.to(torch.int32) - 127)[:, None]).view(-1)


_LR, _BETAS, _EPS, _DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01


def _adamw_plain(s):
    bits, step, (b1, b2) = s["case"]["bits"], s["step"], _BETAS
    g, p = s["g"].float(), s["p"]
    m = _held(s["m"]) if bits == 8 else s["m"]
    v = _held(s["v"]).square() if bits == 8 else s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    root = torch.sqrt(v)
    p.copy_(p * (1 - _LR * _DECAY) - (_LR / (1 - b1 ** step)) * m / (root / math.sqrt(1 - b2 ** step) + _EPS))
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if bits == 8:
        s["m"], s["v"] = _hold(m, False), _hold(root, True)
        return _held(s["m"]).to(torch.bfloat16), _held(s["v"]).to(torch.bfloat16)
    s["m"], s["v"] = m, v
    return m, v


def _pad(a, offsets, cap):
    """a [R, C] by expert -> [E, cap, C], rows behind an expert's last as 0."""
    at = offsets[:-1, None].long() + torch.arange(cap, device=a.device)
    return torch.where((at < offsets[1:, None])[:, :, None], a[at.clamp(max=a.shape[0] - 1)], 0.0)


def _unpad(p, offsets, R):
    """[E, cap, C] -> [R, C]."""
    row = torch.arange(R, device=p.device)
    e = torch.searchsorted(offsets[1:].contiguous(), row, right=True).clamp(max=p.shape[0] - 1)
    return p[e, (row - offsets[e]).clamp(min=0, max=p.shape[1] - 1)]


def _grouped(a, w, offsets, cap):
    """a [R, K] by expert, w [E, N, K] -> [R, N]."""
    return _unpad(torch.bmm(_pad(a, offsets, cap), w.transpose(1, 2).contiguous()), offsets, a.shape[0])


def _exchange_plain(s):
    case, row = s["case"], s["inv_perm"].long()
    T, k, d = case["T"], case["k"], case["d"]
    live = (row < s["offsets"][-1])[:, None]
    dout = s["dout"].float()
    dscale = (torch.where(live, s["y"].float()[row], 0.0).view(T, k, d) * dout[:, None]).sum(2)
    dy = torch.empty_like(s["y"])
    dy[row] = torch.where(live, (s["scale"][:, :, None] * dout[:, None]).view(T * k, d), 0.0).to(dy.dtype)
    dx = torch.where(live, s["dx_perm"].float()[row], 0.0).view(T, k, d).sum(1).to(s["dx_perm"].dtype)
    return {"dy": dy, "dscale": dscale, "dx": dx}


def _adapt_plain(s):
    case, offsets, cap = s["case"], s["offsets"], s["cap"]
    T, k = case["T"], case["k"]
    perm = s["perm_src"].long()
    v = _grouped(s["x"].float()[perm // k], s["a"].float(), offsets, cap)
    delta = _grouped(v, (s["b"].float() * s["adapter_scale"][:, None, None]).transpose(1, 2).contiguous(), offsets, cap)
    at = perm if k == 1 else torch.arange(T * k, device=perm.device)
    live = (torch.arange(T * k, device=perm.device) < offsets[-1])[:, None]
    old = s["y"][at]
    s["y"][at] = torch.where(live, (old.float() + delta).to(old.dtype), old)
    return s["y"]


def _gradient_plain(s):
    case, offsets, cap = s["case"], s["offsets"], s["cap"]
    R, k = case["T"] * case["k"], case["k"]
    perm = s["perm_src"].long()
    dy = s["dy"].float()[perm] if k == 1 else s["dy"].float()
    a, b = s["a"].float(), s["b"].float() * s["adapter_scale"][:, None, None]
    u = _grouped(dy, b, offsets, cap)
    live = (torch.arange(R, device=perm.device) < offsets[-1])[:, None]
    dx = torch.where(live, _grouped(u, a.transpose(1, 2).contiguous(), offsets, cap), 0.0)
    da = torch.bmm(_pad(u, offsets, cap).transpose(1, 2).contiguous(), _pad(s["x"].float()[perm // k], offsets, cap))
    db = torch.bmm(_pad(s["v"], offsets, cap).transpose(1, 2).contiguous(), _pad(dy, offsets, cap)) * s["adapter_scale"][:, None, None]
    rows = torch.empty_like(dx)
    rows[perm if k == 1 else torch.arange(R, device=perm.device)] = dx
    grad = _DT[case["grad"]]
    return {"dx": rows.to(s["x"].dtype), "da": da.to(grad), "db": db.to(grad)}


def run(state):
    case, op = state["case"], state["case"]["op"]
    if op == "adamw":
        state["step"] += 1
    if own:
        import paper_2211_10017_amd as moe
        if op == "adamw":
            t = state["tensors"]
            moe.moe_adamw(t["p"], t["g"], t["m"], t["v"], state["step"], lr=_LR, betas=_BETAS, eps=_EPS, weight_decay=_DECAY, copies=t["copy"])
            m, v = state["m"], state["v"]
            if case["bits"] == 8:
                m, v = moe.moe_adamw_state(*m, torch.bfloat16), moe.moe_adamw_state(*v, torch.bfloat16)
            return {"p": state["p"], "m": m, "v": v, "copy": state["copy"]}
        T, k, offsets = case["T"], case["k"], state["offsets"]
        if op == "exchange":
            active = offsets[case["E"]:]
            dy, dscale = moe.moe_combine_backward(state["dout"], state["y"], state["inv_perm"], state["scale"], active_rows=active)
            return {"dy": dy, "dscale": dscale, "dx": moe.moe_permute_backward(state["dx_perm"], state["inv_perm"], T, k, active_rows=active)}
        index = dict(perm_src=state["perm_src"], k=k, scale=state["adapter_scale"], by_assignment=k == 1)
        if op == "adapt":
            return moe.moe_adapters(state["x"], state["a"], state["b"], offsets, y=state["y"], out=state["y"], **index)
        dx, da, db = moe.moe_adapters_backward(state["dy"], state["x"], state["a"], state["b"], state["v"], offsets, grad_dtype=_DT[case["grad"]], **index)
        return {"dx": dx, "da": da, "db": db}
    if op == "adamw":
        m, v = _adamw_plain(state)
        return {"p": state["p"], "m": m, "v": v, "copy": state["copy"]}
    return {"exchange": _exchange_plain, "adapt": _adapt_plain, "gradient": _gradient_plain}[op](state)


def work(case):
    op = case["op"]
    if op == "adamw":
        n = sum(_starts(case)[1])
        held = 1 + 1 / 32
        states = 16 if case["bits"] == 32 else 4 * held + 2 * (held + 2)              # (8 bits: read back as well)
        return {"bytes": n * (8 + _SIZE[case["g"]] + states + (2 if case["copy"] else 0)), "flops": 0}
    T, k, E = case["T"], case["k"], case["E"]
    live = T - (max(1, round(case["finished"] * T)) if case["finished"] else 0)
    R = live * k
    if op == "exchange":
        d, rows = case["d"], 2
        # dout and dx of every token, y and dx_perm of the active rows, dy of all
        return {"bytes": live * d * _SIZE[case["out"]] + T * d * rows + R * d * (_SIZE[case["y"]] + rows) + T * k * d * _SIZE[case["y"]], "flops": 0}
    K, N, rank = case["K"], case["N"], case["rank"]
    active = E * (1.0 - (1.0 - 1.0 / E) ** R)
    weights = active * rank * (K + N) * 2
    if op == "adapt":
        return {"bytes": live * K * 2 + 2 * R * N * _SIZE[case["y"]] + weights, "flops": 2.0 * R * rank * (K + N)}
    return {"bytes": live * K * 2 + R * N * _SIZE[case["y"]] + T * k * K * 2 + weights + E * rank * (K + N) * _SIZE[case["grad"]] + R * rank * 4,
            "flops": 4.0 * R * rank * (K + N)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------

def _exact_8bit(v, root):
    """The numbers that v stands for when it is held in 8 bits."""
    b = v.reshape(-1, 32)
    top = b.abs().amax(1, keepdim=True)
    unit = torch.ldexp(torch.ones_like(top), torch.where(top > 0, torch.frexp(top)[1] - 8, -127).clamp(min=-127))
    a = b.abs() / unit
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a)[1] - 4).clamp(min=-9))      # three bits behind the leading one, down to 2^-9
    q = torch.round(a / step) * step
    if root:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    return (torch.sign(b) * q * unit).reshape(-1)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "adamw":
        value = lambda h: h[0].view(torch.float8_e4m3fn).double() * torch.exp2(h[1].double() - 127).repeat_interleave(32)  # noqa: E731
        p, g, t, (b1, b2) = s["p"].double(), s["g"].double(), s["step"] + 1, _BETAS
        m, v = (value(s["m"]), value(s["v"]) ** 2) if case["bits"] == 8 else (s["m"].double(), s["v"].double())
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = p - _LR * _DECAY * p - _LR * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + _EPS)
        copy = p if case["copy"] else None
        if case["bits"] == 8:
            m, v = _exact_8bit(m, False), _exact_8bit(torch.sqrt(v), True)
        return {"p": p, "m": m, "v": v, "copy": copy}
    T, k, E = case["T"], case["k"], case["E"]
    R, off = T * k, s["offsets"].tolist()
    perm = s["perm_src"].long()
    token = perm // k
    if op == "exchange":
        n = off[-1]
        d = case["d"]
        rows = s["dout"].double()[token[:n]]
        dy = torch.zeros((R, d), dtype=torch.float64, device="cuda")
        dy[:n] = s["scale"].double().flatten()[perm[:n], None] * rows
        dscale = torch.zeros(R, dtype=torch.float64, device="cuda")
        dscale[perm[:n]] = (rows * s["y"][:n].double()).sum(1)
        dx = torch.zeros((T, d), dtype=torch.float64, device="cuda").index_add_(0, token[:n], s["dx_perm"][:n].double())
        return {"dy": dy, "dscale": dscale.view(T, k), "dx": dx}
    place = perm if k == 1 else torch.arange(R, device="cuda")
    x, scale = s["x"], s["adapter_scale"].double()
    if op == "adapt":
        y = s["y"].double()
    else:
        dx = torch.zeros((R, case["K"]), dtype=torch.float64, device="cuda")
        da, db = (torch.zeros((E, case["rank"], c), dtype=torch.float64, device="cuda") for c in (case["K"], case["N"]))
    for e in range(E):
        at = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        xe, ae, be = x[token[at]].double(), s["a"][e].double(), s["b"][e].double()
        if op == "adapt":
            y[place[at]] += scale[e] * (xe @ ae.T @ be)
            continue
        dye = s["dy"][place[at]].double()
        u = scale[e] * (dye @ be.T)
        dx[place[at]] = u @ ae
        da[e], db[e] = u.T @ xe, scale[e] * ((xe @ ae.T).T @ dye)
    return y if op == "adapt" else {"dx": dx, "da": da, "db": db}
