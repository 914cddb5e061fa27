"""The norm, the activation, the grouped products and their gradients in 64 bits, from their definitions (torch, any device)."""
import math

import torch


def rmsnorm(x, residual, weight, eps):
    h = x.double() if residual is None else x.double() + residual.double()
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + eps)
    w = 1.0 if weight is None else weight.double()
    return h, rstd, h * rstd[:, None] * w


def rmsnorm_backward(dy, h, rstd, weight, dh):
    dy, h, r = dy.double(), h.double(), rstd.double()[:, None]
    g = dy if weight is None else dy * weight.double()
    xhat = h * r
    dx = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
    return dx if dh is None else dx + dh.double(), (dy * xhat).sum(0)


def activation(u, v, scale):
    """a and its derivatives (in u, in v) without the scale; scale [rows]."""
    u = u.double()
    if v is not None:
        p = torch.sigmoid(u)
        return u * p * v.double(), p * (1 + u * (1 - p)) * v.double(), u * p
    P = 0.5 * torch.special.erfc(-u * math.sqrt(0.5))
    return u * P, P + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi), None


def groups(offsets, rows):
    """(first row, rows) of each group: ranges outside [0, rows] and those that start before the end of one before own none."""
    out, reach = [], 0
    for a, b in zip(offsets[:-1], offsets[1:]):
        ok = 0 <= a <= b <= rows
        first, n = (a, b - a) if ok else (0, 0)
        if n and first < reach:
            out.append((0, 0))
        else:
            out.append((first, n))
        if n:
            reach = max(reach, first + n)
    return out


def grouped(form, X, W, owned):
    """(result, sum of the terms' magnitudes) of a grouped product; result rows of no group are NaN (fwd, dgrad)."""
    X = X.double()
    if form == "wgrad":
        W = W.double()
        parts = [(X[a:a + n].T @ W[a:a + n], X[a:a + n].abs().T @ W[a:a + n].abs()) for a, n in owned]
        return torch.stack([p[0] for p in parts]), torch.stack([p[1] for p in parts])
    cols = W.shape[1] if form == "fwd" else W.shape[2]
    out = torch.full((X.shape[0], cols), float("nan"), dtype=torch.float64, device=X.device)
    mag = torch.zeros_like(out)
    for g, (a, n) in enumerate(owned):
        if n:
            w = W[g].double().T if form == "fwd" else W[g].double()
            out[a:a + n], mag[a:a + n] = X[a:a + n] @ w, X[a:a + n].abs() @ w.abs()
    return out, mag


def to_e4m3(x):
    """x rounded to the nearest e4m3 value, ties to even, saturating at 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)
