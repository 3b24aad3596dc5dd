"""Sorted indices, plain implementations in 64 bits and error bounds for what layers are tuned with: the exchange's gradient, adapters and AdamW."""
from __future__ import annotations

import torch

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
U = 2.0 ** -24                                                # half a step of fp32, relative


def half_step(v, dtype):
    """The most that rounding v (64 bits) to dtype moves it: half a step, eps / 2 of the value, and half the smallest number where f16 gives way."""
    return v.abs() * (torch.finfo(dtype).eps / 2) + (2.0 ** -25 if dtype == F16 else 0.0)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def sorted_index(idx, E):
    """perm_src, inv_perm, offsets of expert_idx [T, k] (E: a pruned row), as moe_permute gives them."""
    flat = idx.flatten().long()
    perm = torch.sort(flat, stable=True).indices
    inv = torch.empty_like(perm)
    inv[perm] = torch.arange(len(flat), device=flat.device)
    offsets = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
    offsets[1:] = torch.bincount(flat, minlength=E + 1)[:E].cumsum(0)
    return perm.int(), inv.int(), offsets.int()


def routing(gen, T, k, E, load):
    """load: even | one (a single expert has every row) | ends (the first and the last expert) | none (every row is pruned) | pruned (a third of the tokens)."""
    if load == "one":
        idx = torch.full((T, k), E // 2, device="cuda")
    elif load == "ends":
        idx = torch.randint(0, 2, (T, k), generator=gen, device="cuda") * (E - 1)
    elif load == "none":
        idx = torch.full((T, k), E, device="cuda")
    else:
        idx = torch.randint(0, E, (T, k), generator=gen, device="cuda")
        if load == "pruned":
            idx[torch.rand(T, generator=gen, device="cuda") < 1 / 3] = E
    return idx.int()


def adapters_ref(x, a, b, offsets, perm, k, scale, by_assignment, y, dy=None):
    """out and v of the forward pass, with the sums of the magnitudes of what is added; dx, da, db with dy.  All in 64 bits."""
    R = x.shape[0] if perm is None else perm.numel()
    dev = x.device
    source = torch.arange(R, device=dev) if perm is None else perm.long()
    place = source if by_assignment else torch.arange(R, device=dev)
    (E, rank, K), N = a.shape, b.shape[2]
    off = offsets.tolist()
    z = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)  # noqa: E731
    o = dict(out=z(R, N) if y is None else y.double().clone(), out_mag=z(R, N), v=z(R, rank), v_mag=z(R, rank), dx=z(R, K), dx_mag=z(R, K), da=z(E, rank, K), da_mag=z(E, rank, K),
             db=z(E, rank, N), db_mag=z(E, rank, N))
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        s = 1.0 if scale is None else float(scale[e])
        xe, ae, be = x[source[r] // k].double(), a[e].double(), b[e].double()
        v, vm = xe @ ae.T, xe.abs() @ ae.abs().T
        o["v"][r], o["v_mag"][r] = v, vm
        o["out"][place[r]] += s * (v @ be)
        # v is off by K roundings of sums of this size and, where it goes into products in two 16-bit terms, by 2^-16; the products by `rank` roundings more
        o["out_mag"][place[r]] = abs(s) * ((K + rank + 4) * U * (vm @ be.abs()) + 2.0 ** -16 * (v.abs() @ be.abs()))
        if dy is None:
            continue
        d = dy[place[r]].double()
        n = off[e + 1] - off[e]
        u, um = s * (d @ be.T), abs(s) * (d.abs() @ be.abs().T)
        o["dx"][place[r]] = u @ ae
        o["dx_mag"][place[r]] = (N + rank + 4) * U * (um @ ae.abs()) + 2.0 ** -16 * (u.abs() @ ae.abs())
        o["da"][e], o["da_mag"][e] = u.T @ xe, (N + n + 4) * U * (um.T @ xe.abs()) + 2.0 ** -16 * (u.abs().T @ xe.abs())
        o["db"][e], o["db_mag"][e] = s * (v.T @ d), abs(s) * ((K + n + 4) * U * (vm.T @ d.abs()) + 2.0 ** -16 * (v.abs().T @ d.abs()))
    return o


def within(got, want, slack):
    """got (rounded to its type) is want up to `slack` and the rounding."""
    w = want.double()
    assert got.shape == w.shape and bool(torch.isfinite(got.float()).all())
    off = (got.double() - w).abs()
    most = slack + half_step(w.abs() + slack, got.dtype)
    assert bool((off <= most).all()), "off by %.3g where %.3g is allowed" % tuple(float(t.flatten()[((off - most).flatten().argmax())]) for t in (off, most))
