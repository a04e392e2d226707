"""Plain definitions, in 64 bits on the CPU, of the calls between and behind a layer's halves."""
from __future__ import annotations

import math

import torch

MASK = 0xFFFFFFFF


def philox(counter, key):
    """Four words of Philox4x32 with ten rounds."""
    a, b, c, d = counter
    k0, k1 = key
    for _ in range(10):
        p, q = 0xD2511F53 * a, 0xCD9E8D57 * c
        a, b, c, d = (q >> 32) ^ b ^ k0, q & MASK, (p >> 32) ^ d ^ k1, p & MASK
        k0, k1 = (k0 + 0x9E3779B9) & MASK, (k1 + 0xBB67AE85) & MASK
    return a, b, c, d


def factors(T, d, p, seed, step, site):
    """[T, d]: what every element is multiplied with."""
    below = round(65536 * p)
    out = torch.ones((T, d), dtype=torch.float64)
    if not below:
        return out
    runs = -(-d // 8)
    for t in range(T):
        for j in range(runs):
            n = t * runs + j
            words = philox((n & MASK, n >> 32, site & MASK, step & MASK), (seed & MASK, seed >> 32 & MASK))
            for i in range(min(8, d - 8 * j)):
                u = words[i // 2] >> 16 * (i % 2) & 0xFFFF
                out[t, 8 * j + i] = 0.0 if u < below else 65536 / (65536 - below)
    return out


def dropped(x, f):
    """What a dropped element holds has no effect."""
    return torch.where(f == 0, 0.0, x.double() * f)


def norm(x, residual, weight, eps, f):
    """H, Y"""
    h = dropped(x, f)
    if residual is not None:
        h = h + residual.double()
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return h, y if weight is None else y * weight.double()


def norm_back(dy, h, weight, eps, dh, f):
    """dX, dR, dW"""
    dy, h = dy.double(), h.double()
    r = torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    n, g = h / r, dy if weight is None else dy * weight.double()
    out = (g - n * (g * n).mean(-1, keepdim=True)) / r
    if dh is not None:
        out = out + dh.double()
    return dropped(out, f), out, (dy * n).sum(0)


def vocab_loss(X, W, targets, weights=None):
    """loss, lse, dX, dW; tokens whose target is no row of W take no part."""
    T, V = X.shape[0], W.shape[0]
    loss, lse = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    dX, dW = torch.zeros(X.shape, dtype=torch.float64), torch.zeros(W.shape, dtype=torch.float64)
    held = [t for t in range(T) if 0 <= int(targets[t]) < V]
    if not held:
        return loss, lse, dX, dW
    x, w = X[held].double(), W.double()
    t = targets[held].long()
    z = x @ w.t()
    at = torch.arange(len(held))
    others = z.clone()
    others[at, t] = -math.inf
    ahead = torch.logsumexp(others, -1) - z[at, t]           # of all others together, ahead of the target
    lse[held] = torch.logsumexp(z, -1)
    loss[held] = torch.clamp(ahead, min=0) + torch.log1p(torch.exp(-ahead.abs()))
    G = torch.exp(z - lse[held][:, None])
    G[at, t] = -1 / (1 + torch.exp(-ahead))
    if weights is not None:
        G = G * weights[held].double()[:, None]
    dX[held] = G @ w
    return loss, lse, dX, G.t() @ x
