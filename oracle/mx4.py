"""The microscaled 4-bit format, its grouped product and the router's balance loss in 64 bits, from their definitions (numpy; test infrastructure only)."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def exponents(v):
    """Whole exponents of the blocks' scales, [R, K/32]; 128 for a block that is not a number."""
    a = np.abs(v.reshape(v.shape[0], -1, 32)).max(axis=2)
    e = np.full(a.shape, -127, dtype=np.int64)
    ok = np.isfinite(a)
    _, ex = np.frexp(np.where(ok, a, 1.0))                 # a = m 2^ex, m in [0.5, 1): floor(log2 a) = ex - 1
    e = np.where(a > 0, np.maximum(ex - 3, -127), e)
    return np.where(ok, e, 128)


def nearest_code(a):
    """Index into GRID of the number nearest to a >= 0, ties to the even index, at most 7."""
    half = (GRID[1:] + GRID[:-1]) / 2
    i = np.searchsorted(half, a, side="left")              # halfway: the lower index ...
    tie = (i < 7) & (half[np.minimum(i, 6)] == a) & (i % 2 == 1)
    return np.where(tie, i + 1, i)                         # ... unless it is odd


def quantize(v, e=None):
    """v [R, K] -> (codes uint8 [R, K/2], scales uint8 [ceil(K/128), R, 4], values float64 [R, K])."""
    v = np.asarray(v, dtype=np.float64)
    R, K = v.shape
    e = exponents(v) if e is None else e
    wide = np.repeat(e, 32, axis=1)
    unit = np.ldexp(1.0, np.minimum(wide, 127))
    with np.errstate(invalid="ignore"):
        i = np.where(wide == 128, 0, nearest_code(np.where(wide == 128, 0.0, np.abs(v) / unit)))
    neg = np.signbit(v) & (wide != 128)
    code = (i + 8 * neg).astype(np.uint8)
    scales = np.zeros((R, -(-K // 128) * 4), dtype=np.uint8)
    scales[:, :K // 32] = e + 127
    values = np.where(wide == 128, np.nan, np.where(neg, -1.0, 1.0) * GRID[i] * unit)
    return code[:, 0::2] | (code[:, 1::2] << 4), np.ascontiguousarray(scales.reshape(R, -1, 4).transpose(1, 0, 2)), values


def dequantize(codes, scales):
    R, half = codes.shape
    c = np.empty((R, 2 * half), dtype=np.int64)
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    s = scales.transpose(1, 0, 2).reshape(R, -1)[:, :half // 16].astype(np.int64)
    unit = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return np.where(c > 7, -1.0, 1.0) * GRID[c & 7] * np.repeat(unit, 32, axis=1)


def gelu(v):
    from scipy.special import ndtr
    return v * ndtr(v)


ACTIVATIONS = {None: lambda v: v, "relu": lambda v: np.maximum(v, 0.0), "gelu": gelu}


def product(a, offsets, w, bias=None):
    """a [R, K], w [E, N, K] in 64 bits -> (y [R, N], sum of the terms' magnitudes [R, N]); rows past the last expert's are NaN."""
    R, N = a.shape[0], w.shape[1]
    y, size = np.full((R, N), np.nan), np.zeros((R, N))
    for e in range(w.shape[0]):
        r = slice(offsets[e], offsets[e + 1])
        y[r], size[r] = a[r] @ w[e].T, np.abs(a[r]) @ np.abs(w[e]).T
        if bias is not None:
            y[r] += bias[e]
            size[r] += np.abs(bias[e])
    return y, size


def balance(logits, idx, coef, renormalize, dloss=0.0, dscale=None):
    """loss, counts, prob_mean, scale, weight and the gradient of dloss * loss + sum(dscale * scale) with respect to the logits, by the chain rule
    through p and the softmax's whole Jacobian."""
    z = np.asarray(logits, dtype=np.float64)
    T, E = z.shape
    k = idx.shape[1]
    with np.errstate(invalid="ignore"):
        top = z.max(axis=1, keepdims=True, initial=-np.inf)
        ex = np.where(np.isneginf(z), 0.0, np.exp(z - np.where(np.isneginf(top), 0.0, top)))
    total = ex.sum(axis=1, keepdims=True)
    p = ex / np.where(total == 0, 1.0, total)
    used = (idx >= 0) & (idx < E)
    at = np.where(used, idx, 0)
    chosen = np.where(used, np.take_along_axis(p, at, 1), 0.0)
    live = used.any(axis=1)
    counts = np.bincount(idx[used], minlength=E)[:E]
    A, N = max(1, counts.sum()), max(1, live.sum())
    mean = p[live].sum(axis=0) / N
    weight = coef * E * counts / A / N
    loss = coef * E * (counts / A * mean).sum()
    ds = np.zeros((T, k)) if dscale is None else np.where(used, dscale, 0.0)
    if renormalize and k > 1:
        s = chosen.sum(axis=1, keepdims=True)
        s = np.where(s == 0, 1.0, s)
        # d scale_j / d chosen_j = (s - chosen_j) / s^2, the other chosen ones together: exactly 0 for a token with one expert
        others = np.stack([np.delete(chosen, j, axis=1).sum(axis=1) for j in range(k)], axis=1)
        passed = np.stack([np.delete(ds * chosen, j, axis=1).sum(axis=1) for j in range(k)], axis=1)
        scale, dchosen = chosen / s, (ds * others - passed) / s ** 2
    else:
        scale, dchosen = chosen, ds
    dp = dloss * weight[None, :] * live[:, None]
    for j in range(k):
        np.add.at(dp, (np.arange(T), at[:, j]), np.where(used[:, j], dchosen[:, j], 0.0))
    grad = np.where(live[:, None], p * (dp - (p * dp).sum(axis=1, keepdims=True)), 0.0)
    size = p * (np.abs(dp) + (p * np.abs(dp)).sum(axis=1, keepdims=True))
    return dict(loss=loss, counts=counts, prob_mean=mean, scale=scale, weight=weight, dlogits=grad, size=size)
