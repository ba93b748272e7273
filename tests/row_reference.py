"""Plain 64-bit forms of the operators on the rows of many parts (numpy and torch float64 on the CPU)."""
import math

import numpy as np
import torch

F64 = torch.float64


def mask(seed, ids, d, p):
    """(kept [n, d] of truth values, scale)."""
    t = math.floor(65536 * p + 0.5)

    def step(z):
        z = (z + np.uint64(0x9E3779B97F4A7C15))
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        key = step(np.array([seed % 2**64], dtype=np.uint64))[0]
        rows = np.asarray(ids, dtype=np.int64).astype(np.uint64) & np.uint64(0xFFFFFFFF)
        col = np.arange(d, dtype=np.uint64)
        word = step(key ^ ((rows[:, None] << np.uint64(32)) | (col // np.uint64(4))[None, :]))
        lane = (word >> (np.uint64(16) * (col % np.uint64(4)))[None, :]) & np.uint64(0xFFFF)
    return torch.from_numpy(lane.astype(np.int64) >= t), 65536.0 / (65536 - t) if t < 65536 else 0.0


def dropout(x, p, seed, ids=None):
    kept, scale = mask(seed, np.arange(x.shape[0]) if ids is None else ids, x.shape[1], p)
    return torch.where(kept, x.to(F64) * scale, torch.zeros((), dtype=F64))


def linear(X, offsets, W, b=None):
    """[n, d_out]; rows of no part are zero.  W, b with a leading part dimension or without."""
    n, d_out = X.shape[0], W.shape[-1]
    y = X.new_zeros(n, d_out, dtype=F64)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        w = (W[g] if W.dim() == 3 else W).to(F64)
        y[lo:hi] = X[lo:hi].to(F64) @ w
        if b is not None:
            y[lo:hi] += (b[g] if b.dim() == 2 else b).to(F64)
    return y


def linear_dw(X, dY, offsets):
    dw = torch.stack([X[a:b].to(F64).T @ dY[a:b].to(F64) for a, b in zip(offsets, offsets[1:])])
    return dw, torch.stack([dY[a:b].to(F64).sum(0) for a, b in zip(offsets, offsets[1:])])


def group_norm(X, offsets, groups, gamma, beta, scope, act, slope, eps, kept=None, scale=1.0):
    """Differentiable in X, gamma, beta, slope (all float64, gamma, beta [G, C], slope [G]); returns (Y, stats, U, xhat), rows of
    no part zero."""
    n, C = X.shape
    ys, stats, us, xs = [], [], [], []
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        x = X[lo:hi].reshape(hi - lo, groups, C // groups)
        over = (2,) if scope == "row" else (0, 2)
        if hi > lo:
            mean = x.mean(dim=over, keepdim=True)
            var = ((x - mean) ** 2).mean(dim=over, keepdim=True)
        else:
            mean = x.new_zeros(0 if scope == "row" else 1, groups, 1)
            var = mean
        rstd = 1 / torch.sqrt(var + eps)
        stats.append(torch.stack([mean.reshape(-1, groups), rstd.reshape(-1, groups)], dim=2))
        xhat = ((x - mean) * rstd).reshape(hi - lo, C)
        u = xhat * gamma[g] + beta[g]
        if act == "relu":
            h = torch.where(u > 0, u, torch.zeros_like(u))
        elif act == "prelu":
            h = torch.where(u > 0, u, u * slope[g])
        elif act == "silu":
            h = u * torch.sigmoid(u)
        else:
            h = u
        if kept is not None:
            h = torch.where(kept[lo:hi], h * scale, torch.zeros_like(h))
        ys.append(h)
        us.append(u)
        xs.append(xhat)
    pad = lambda parts: torch.cat([X.new_zeros(offsets[0], C), *parts, X.new_zeros(n - offsets[-1], C)])  # noqa: E731
    return pad(ys), torch.cat(stats), pad(us), pad(xs)
