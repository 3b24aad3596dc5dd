"""Operators beside the expert layer, for timing: microscaled 4-bit floating point (quantisation, grouped product, expert FFN) and the
router's balance loss with its gradient.  `run` calls them as users do, or, with `own` false, computes them in elementary torch operations.

The sizes are those of this repository's configurations, tests and benchmark (d_model 512 to 4096, d_ff four times that, 8 to 128 experts,
1 to 16384 tokens) and generic ones beside them."""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _rows(name=None, **kw):
    case = dict(op="rows", R=64, K=1024, dtype="f16")
    case.update(kw)
    return dict(name=name, **case) if name else case


def _experts(name=None, **kw):
    case = dict(op="experts", E=32, K=1024, N=4096)
    case.update(kw)
    return dict(name=name, **case) if name else case


def _product(name=None, **kw):
    case = dict(op="product", T=64, k=2, E=32, K=1024, N=4096, out="f16", bias=False, load="even")
    case.update(kw)
    return dict(name=name, **case) if name else case


def _ffn(name=None, **kw):
    case = dict(op="ffn", T=64, k=2, E=32, d=1024, F=4096, dtype="f16", activation="relu", bias=False, load="even", finished=0.0)
    case.update(kw)
    return dict(name=name, **case) if name else case


def _router(name=None, **kw):
    case = dict(op="router", T=64, k=2, E=32, dtype="f32", renormalize=True, load="even", finished=0.0)
    case.update(kw)
    return dict(name=name, **case) if name else case


def listed():
    return [
        # the rows of a decoder batch before they meet 4-bit experts: launches and latency
        _rows("rows_64_f16"),
        # the rows of the largest batch, bf16
        _rows("rows_16384_bf16", R=16384, K=4096, dtype="bf16"),
        # loading a model: one weight tensor of the paper's layer from its fp32 masters
        _experts("experts_32"),
        # Table 1 of the paper: one grouped product of about 40 decoder tokens, one expert each
        _product("product_40", T=40, k=1, out="f32"),
        # a grouped product of an encoder batch over many experts, some of them busier than others
        _product("product_4096", T=4096, E=128, K=2048, N=8192, load="uneven"),
        # one sentence, one decoder step: the FFN's smallest call
        _ffn("ffn_1", T=1),
        # the benchmark's headline batch: 64 tokens, two of 32 experts, a quarter of the sentences already ended
        _ffn("ffn_64", finished=0.25),
        # a ragged encoder batch in bf16 with biases and GELU, feature counts that are odd multiples of 64
        _ffn("ffn_997_bf16", T=997, E=16, d=704, F=2880, dtype="bf16", activation="gelu", bias=True, load="uneven"),
        # the largest layer
        _ffn("ffn_8192", T=8192, E=64, d=4096, F=16384),
        # one decoder batch's router step
        _router("router_64"),
        # tuning a router: an encoder batch, bf16 logits, unevenly loaded experts, one expert per token
        _router("router_16384_bf16", T=16384, k=1, E=64, dtype="bf16", renormalize=False, load="uneven"),
        # a large training batch over many experts
        _router("router_131072", T=131072, E=256),
    ]


_SHAPES = [(512, 2048), (704, 2880), (1024, 4096), (2048, 8192), (4096, 16384)]
_MAX_FLOPS = 4.3e12              # the largest listed case
_MAX_ELEMENTS = 64 * 4096 * 16384


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows", "experts", "product", "product", "ffn", "ffn", "ffn", "router", "router"])
    load = rng.choice(["even", "even", "uneven"])
    if kind == "rows":
        K = 64 * _log_int(rng, 1, 256)
        return _rows(R=_log_int(rng, 1, min(16384, (1 << 26) // K)), K=K, dtype=rng.choice(["f16", "bf16", "f32"]))
    if kind == "experts":
        K, N = 64 * _log_int(rng, 1, 256), 32 * _log_int(rng, 1, 256)
        return _experts(E=_log_int(rng, 1, max(1, min(128, (1 << 27) // (K * N)))), K=K, N=N)
    if kind == "product":
        while True:
            T, k, E = _log_int(rng, 1, 8192), rng.choice([1, 2]), rng.choice([2, 8, 16, 32, 64, 128])
            K, N = 64 * _log_int(rng, 2, 128), 32 * _log_int(rng, 4, 256)
            if 2.0 * T * k * K * N <= _MAX_FLOPS / 4 and E * K * N <= _MAX_ELEMENTS / 2:
                return _product(T=T, k=k, E=E, K=K, N=N, out=rng.choice(["f16", "bf16", "f32"]), bias=rng.random() < 0.3, load=load)
    if kind == "ffn":
        decode = rng.random() < 0.5
        while True:
            T = _log_int(rng, 1, 256) if decode else _log_int(rng, 257, 8192)
            k, E = rng.choice([1, 2]), rng.choice([8, 16, 32, 64, 128])
            d, F = rng.choice(_SHAPES)
            if 4.0 * T * k * d * F <= _MAX_FLOPS and E * d * F <= _MAX_ELEMENTS:
                break
        return _ffn(T=T, k=k, E=E, d=d, F=F, dtype=rng.choice(["f16", "bf16"]), activation=rng.choice(["relu", "relu", "gelu"]),
                    bias=rng.random() < 0.3, load=load, finished=rng.choice([0.0, rng.uniform(0.1, 0.6)]) if decode and T > 8 else 0.0)
    E = rng.choice([8, 16, 32, 61, 64, 100, 128, 160, 256])
    return _router(T=_log_int(rng, 1, 131072), k=rng.choice([1, 2]), E=E, dtype=rng.choice(["f32", "f16", "bf16"]),
                   renormalize=rng.random() < 0.5, load=load, finished=rng.choice([0.0, 0.0, rng.uniform(0.1, 0.6)]))


# ---- the plain form: elementary operations in 32 bits -----------------------------------------------------------------------------

def _pow2(e):
    """2^e in fp32, for whole -127 <= e <= 127, put together from its bits (2^-127 is a subnormal number)."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _split(v):
    """v [.., K] -> blocks of 32 of it, as the nearest e2m1 numbers and the whole exponents they are in units of (128: not a number)."""
    b = v.float().unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    e = ((amax.view(torch.int32) >> 23) - 129).clamp(-127, 127)          # floor(log2 amax) - 2; of subnormal amax the clamp decides
    a = (b * _pow2(-e)).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = torch.copysign((torch.round(a / step) * step).clamp(max=6.0), b)
    fine = amax < math.inf
    return torch.where(fine, q, 0.0), torch.where(fine, e, 128)


def _values(q, e):
    return torch.where(e < 128, q * _pow2(e.clamp(max=127)), math.nan).flatten(-2)


def _pack(q, e):
    """The 4-bit format: codes [.., R, K / 2], even k in the low nibble, and scales [.., ceil(K / 128), R, 4]."""
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    code = code.flatten(-2)
    codes = code[..., 0::2] | (code[..., 1::2] << 4)
    s = (e.squeeze(-1) + 127).to(torch.uint8)                            # [.., R, K / 32]
    s = torch.nn.functional.pad(s, (0, -s.shape[-1] % 4)).unflatten(-1, (-1, 4))
    return codes, s.transpose(-2, -3).contiguous()


def _unpack(codes, scales):
    K = codes.shape[-1] * 2
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    m = (c & 7).float()
    v = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, m * 2 - 8))
    v = torch.where(c > 7, -v, v).unflatten(-1, (-1, 32))
    s = scales.transpose(-2, -3).flatten(-2)[..., :K // 32].unsqueeze(-1).to(torch.int32) - 127
    return _values(v, s)


def _gelu(v):
    return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))


def _grouped(a, w, offsets, cap):
    """a [R, K] by expert, w [E, N, K] -> [R, N]: the rows of an expert as one matrix of `cap` rows, the most that any has."""
    R = a.shape[0]
    at = offsets[:-1, None].long() + torch.arange(cap, device=a.device)
    x = a[at.clamp(max=R - 1)]                                           # [E, cap, K]
    y = torch.bmm(w, x.transpose(1, 2).contiguous())                     # [E, N, cap]
    row = torch.arange(R, device=a.device)
    e = torch.searchsorted(offsets[1:].contiguous(), row, right=True).clamp(max=w.shape[0] - 1)
    return y.transpose(1, 2)[e, (row - offsets[e]).clamp(max=cap - 1)]


def _of_row(bias, offsets, R):
    row = torch.arange(R, device=bias.device)
    return bias[torch.searchsorted(offsets[1:].contiguous(), row, right=True).clamp(max=bias.shape[0] - 1)].float()


def _router_plain(s):
    logits, idx, E = s["logits"].float(), s["idx"].long(), s["case"]["E"]
    ex = torch.exp(logits - logits.amax(1, keepdim=True))
    p = ex / ex.sum(1, keepdim=True)
    used = idx < E
    chosen = torch.where(used, p.gather(1, idx.clamp(max=E - 1)), 0.0)
    renorm = s["case"]["renormalize"] and idx.shape[1] > 1
    total = chosen.sum(1, keepdim=True) if renorm else torch.ones_like(chosen[:, :1])
    scale = torch.where(used, chosen / torch.where(total > 0, total, 1.0), 0.0)
    counts = torch.zeros(E + 1, dtype=torch.int32, device=p.device)
    counts.index_add_(0, idx.flatten(), torch.ones_like(idx.flatten(), dtype=torch.int32))
    counts = counts[:E]
    live = used.any(1, keepdim=True)
    A, N = counts.sum().clamp(min=1).float(), live.sum().clamp(min=1).float()
    mean = torch.where(live, p, 0.0).sum(0) / N
    w = s["coef"] * E * counts.float() / (A * N)
    loss = (w * mean).sum() * N
    dl = s["dloss"] * p * (w - (p * w).sum(1, keepdim=True))
    ds = torch.where(used, s["dscale"], 0.0)
    if renorm:
        dl.scatter_add_(1, idx.clamp(max=E - 1), scale * (ds - (scale * ds).sum(1, keepdim=True)))
    else:
        dl -= p * (scale * ds).sum(1, keepdim=True)
        dl.scatter_add_(1, idx.clamp(max=E - 1), scale * ds)
    dl = torch.where(live, dl, 0.0)
    return {"loss": loss, "counts": counts, "prob_mean": mean, "scale": scale, "dlogits": dl.to(s["logits"].dtype)}


# ---- inputs -----------------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _activations(gen, T, d):
    """Rows as layers see them: normally distributed, with channels of unlike size."""
    return torch.randn((T, d), generator=gen, device="cuda") * torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda"))


def _logits(gen, T, E, load):
    l = torch.randn((T, E), generator=gen, device="cuda").mul_(0.64)
    return l + (torch.rand(E, generator=gen, device="cuda") - 0.5) * 0.36 if load == "uneven" else l


def _routing(gen, case):
    """Sorted routing index of a batch: perm_src, expert_offsets and the most rows that an expert has."""
    T, k, E = case["T"], case["k"], case["E"]
    idx = _logits(gen, T, E, case["load"]).topk(k, dim=1).indices
    if case.get("finished"):
        idx[torch.randperm(T, generator=gen, device="cuda")[:max(1, round(case["finished"] * T))]] = E
    flat = idx.flatten()
    perm = torch.sort(flat, stable=True).indices.to(torch.int32)
    counts = torch.bincount(flat, minlength=E + 1)[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = counts.cumsum(0)
    return perm, offsets, max(1, int(counts.max()))


def _weights(gen, E, K, N):
    """An expert matrix after the other, as a checkpoint in the 4-bit format brings them."""
    codes = torch.empty((E, N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((E, -(-K // 128), N, 4), dtype=torch.uint8, device="cuda")
    for e in range(E):
        codes[e], scales[e] = _pack(*_split(torch.randn((N, K), generator=gen, device="cuda").mul_(0.02)))
    return codes, scales


def _bias(gen, E, N, wanted):
    return torch.randn((E, N), generator=gen, device="cuda").mul_(0.02).half() if wanted else None


def prepare(case, seed):
    gen, op = _gen(seed), case["op"]
    s = {"case": case}
    if op == "rows":
        s["x"] = _activations(gen, case["R"], case["K"]).to(_DT[case["dtype"]])
    elif op == "experts":
        s["w"] = torch.randn((case["E"], case["K"], case["N"]), generator=gen, device="cuda").mul_(0.02)
    elif op == "product":
        s["perm_src"], s["offsets"], s["cap"] = _routing(gen, case)
        s["a"] = _pack(*_split(_activations(gen, case["T"], case["K"])))
        s["w"] = _weights(gen, case["E"], case["K"], case["N"])
        s["b"] = _bias(gen, case["E"], case["N"], case["bias"])
    elif op == "ffn":
        s["perm_src"], s["offsets"], s["cap"] = _routing(gen, case)
        s["x"] = _activations(gen, case["T"], case["d"]).to(_DT[case["dtype"]])
        s["w1"], s["w2"] = _weights(gen, case["E"], case["d"], case["F"]), _weights(gen, case["E"], case["F"], case["d"])
        s["b1"], s["b2"] = _bias(gen, case["E"], case["F"], case["bias"]), _bias(gen, case["E"], case["d"], case["bias"])
        # rows of finished sentences stand behind the others; a call writes none of them
        s["y"] = torch.zeros((case["T"] * case["k"], case["d"]), dtype=_DT[case["dtype"]], device="cuda")
    else:
        T, k, E = case["T"], case["k"], case["E"]
        s["logits"] = _logits(gen, T, E, case["load"]).to(_DT[case["dtype"]])
        s["idx"] = s["logits"].float().topk(k, dim=1).indices.to(torch.int32)
        if case["finished"]:
            s["idx"][torch.randperm(T, generator=gen, device="cuda")[:round(case["finished"] * T)]] = E
        s["dscale"] = torch.randn((T, k), generator=gen, device="cuda") * 1e-2
        s["dloss"] = torch.ones((), device="cuda")
        s["coef"] = 0.01
    return s


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        import paper_2211_10017_amd as moe
        if op == "rows":
            return moe.moe_mx4_dequantize(*moe.moe_mx4_quantize_rows(state["x"]), torch.bfloat16)
        if op == "experts":
            return moe.moe_mx4_dequantize(*moe.moe_mx4_quantize_experts(state["w"]), torch.bfloat16)
        if op == "product":
            return moe.moe_grouped_gemm_mx4(*state["a"], state["offsets"], *state["w"], bias=state["b"], perm_src=state["perm_src"],
                                            k=case["k"], y_dtype=_DT[case["out"]], max_rows_per_expert=case["T"])
        if op == "ffn":
            return moe.moe_grouped_ffn_mx4(state["x"], state["offsets"], *state["w1"], *state["w2"], b1=state["b1"], b2=state["b2"],
                                           perm_src=state["perm_src"], k=case["k"], activation=case["activation"], y_perm=state["y"],
                                           max_rows_per_expert=case["T"])
        loss, counts, mean, scale, weight = moe.moe_balance_loss(state["logits"], state["idx"], state["coef"], case["renormalize"])
        dlogits = moe.moe_balance_loss_backward(state["logits"], state["idx"], weight, state["dloss"], state["dscale"], case["renormalize"])
        return {"loss": loss, "counts": counts, "prob_mean": mean, "scale": scale, "dlogits": dlogits}
    if op == "rows":
        return _values(*_split(state["x"])).to(torch.bfloat16)
    if op == "experts":
        return _values(*_split(state["w"].transpose(1, 2))).to(torch.bfloat16)
    if op == "router":
        return _router_plain(state)
    offsets, cap, R = state["offsets"], state["cap"], case["T"] * case["k"]
    source = state["perm_src"].long() // case["k"]
    if op == "product":
        y = _grouped(_unpack(*state["a"])[source], _unpack(*state["w"]), offsets, cap)
        return (y if state["b"] is None else y + _of_row(state["b"], offsets, R)).to(_DT[case["out"]])
    h = _grouped(_values(*_split(state["x"]))[source], _unpack(*state["w1"]), offsets, cap)
    h = h if state["b1"] is None else h + _of_row(state["b1"], offsets, R)
    h = _values(*_split(torch.relu(h) if case["activation"] == "relu" else _gelu(h)))
    y = _grouped(h, _unpack(*state["w2"]), offsets, cap)
    y = y if state["b2"] is None else y + _of_row(state["b2"], offsets, R)
    return torch.where(torch.arange(R, device="cuda")[:, None] < offsets[-1], y, 0.0).to(_DT[case["dtype"]])


def _active(case):
    """Experts that rows reach: all that a draw of T * k assignments is expected to touch."""
    E, R = case["E"], (case["T"] - round(case.get("finished", 0.0) * case["T"])) * case["k"]
    return E * (1.0 - (1.0 - 1.0 / E) ** R)


def work(case):
    op = case["op"]
    size = {"f16": 2, "bf16": 2, "f32": 4}
    held = 0.5 + 1.0 / 32                                                # bytes of a value in the 4-bit format
    if op == "rows":
        return {"bytes": case["R"] * case["K"] * (size[case["dtype"]] + held + 2), "flops": 0}
    if op == "experts":
        return {"bytes": case["E"] * case["K"] * case["N"] * (4 + held + 2), "flops": 0}
    if op == "router":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": 2 * T * E * size[case["dtype"]] + 12 * T * k, "flops": 0}
    live = case["T"] - round(case.get("finished", 0.0) * case["T"])
    R = live * case["k"]
    if op == "product":
        K, N = case["K"], case["N"]
        return {"bytes": _active(case) * (K * N * held + (2 * N if case["bias"] else 0)) + live * K * held + R * N * size[case["out"]],
                "flops": 2.0 * R * K * N}
    d, F = case["d"], case["F"]
    return {"bytes": _active(case) * (2 * d * F * held + (2 * (d + F) if case["bias"] else 0)) + live * d * 2 + R * d * 2,
            "flops": 4.0 * R * d * F}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------------

def _exact_mx(v):
    """The values that v [R, K] stands for in the 4-bit format, by a search among the halfway points of its numbers."""
    R, K = v.shape
    v = v.double().reshape(R, K // 32, 32)
    top = v.abs().amax(2, keepdim=True)
    _, ex = torch.frexp(top)                                             # top = m 2^ex with m in [0.5, 1)
    unit = torch.ldexp(torch.ones_like(top), torch.where(top > 0, ex - 3, -127).clamp(-127, 127))
    a = v.abs() / unit
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=v.device)
    half = (grid[1:] + grid[:-1]) / 2
    up = torch.searchsorted(half, a)                                     # halfway goes down, ...
    up = torch.where((up < 7) & (half[up.clamp(max=6)] == a) & (up % 2 == 1), up + 1, up)      # ... unless the code above is the even one
    return (torch.sign(v) * grid[up] * unit).reshape(R, K)


def _exact_held(codes, scales):
    """Values of codes [N, K / 2] and scales [G, N, 4]."""
    N, half = codes.shape
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=codes.device)
    v = torch.empty((N, half * 2), dtype=torch.float64, device=codes.device)
    v[:, 0::2], v[:, 1::2] = grid[(codes % 16).int()], grid[(codes // 16).int()]
    s = scales.permute(1, 0, 2).reshape(N, -1)[:, :half // 16].double()
    return v * torch.exp2(s - 127).repeat_interleave(32, dim=1)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "rows":
        return _exact_mx(s["x"])
    if op == "experts":
        return torch.stack([_exact_mx(s["w"][e].T.contiguous()) for e in range(case["E"])])
    if op == "router":
        T, k, E = case["T"], case["k"], case["E"]
        z, idx = s["logits"].double(), s["idx"].long()
        p = torch.softmax(z, 1)
        p1 = torch.cat([p, torch.zeros_like(p[:, :1])], 1)               # (index E: a finished sentence)
        hot = torch.nn.functional.one_hot(idx, E + 1).double()           # [T, k, E + 1]
        live = (idx < E).any(1).double()
        c, N = hot.sum((0, 1))[:E], max(1.0, float(live.sum()))
        A = max(1.0, float(c.sum()))
        mean = (p * live[:, None]).sum(0) / N
        g = torch.zeros_like(p1)                                         # dL / dp
        g[:, :E] = s["coef"] * E * c / A / N * live[:, None]
        chosen = p1.gather(1, idx)
        ds = s["dscale"].double()
        if case["renormalize"] and k > 1:
            t = chosen.sum(1, keepdim=True).clamp(min=1e-300)
            scale = chosen / t
            dchosen = ds / t - (ds * chosen).sum(1, keepdim=True) / t ** 2
        else:
            scale, dchosen = chosen, ds
        g = (g + (hot * dchosen[:, :, None]).sum(1))[:, :E] * live[:, None]
        return {"loss": s["coef"] * E * (c / A * mean).sum(), "counts": None, "prob_mean": mean, "scale": scale,
                "dlogits": p * (g - (p * g).sum(1, keepdim=True))}
    R, k = case["T"] * case["k"], case["k"]
    off = s["offsets"].tolist()
    token = s["perm_src"].long() // k
    y = torch.zeros((R, case["N"] if op == "product" else case["d"]), dtype=torch.float64, device="cuda")
    a = _exact_held(*s["a"]) if op == "product" else _exact_mx(s["x"])
    for e in range(case["E"]):
        lo, hi = off[e], off[e + 1]
        if lo == hi:
            continue
        h = a[token[lo:hi]]
        for w, b, last in ([("w", "b", True)] if op == "product" else [("w1", "b1", False), ("w2", "b2", True)]):
            h = h @ _exact_held(s[w][0][e], s[w][1][e]).T
            if s[b] is not None:
                h = h + s[b][e].double()
            if not last:
                h = h.clamp(min=0) if case["activation"] == "relu" else h * torch.special.ndtr(h)
                h = _exact_mx(h)
        y[lo:hi] = h
    return y
