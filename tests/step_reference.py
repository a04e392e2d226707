"""Plain definitions, in 64 bits on the CPU, of the calls around attention and the gradients."""
from __future__ import annotations

import math

import torch


def rope(x, table, positions, interleaved, inverse):
    """x [B,H,S,D]; table [n_pos, rot]; positions [B,S]."""
    x, table = x.double(), table.double()
    rot = table.shape[1]
    h = rot // 2
    out = x.clone()
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = table[positions.long(), i][:, None], table[positions.long(), h + i][:, None]
        if inverse:
            s = -s
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., a] * s + x[..., b] * c
    return out


def rope_frequencies(rot, base, kind, factor, trained, low, high):
    f = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if kind == 2 else base
        v = b ** (-2 * i / rot)
        if kind == 1:
            v /= factor
        if kind == 3:
            g = min(max((trained * v / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            v = v * g + v / factor * (1 - g)
        f.append(v)
    return f


def key_ranges(B, S, docs, causal):
    """docs: [(begin, end, prefix)] over B*S tokens."""
    lo, hi = torch.zeros((B, S), dtype=torch.int32), torch.zeros((B, S), dtype=torch.int32)
    for x, y, p in docs:
        for t in range(x, y):
            b, s = divmod(t, S)
            first, end = max(x - b * S, 0), min(y - b * S, S)
            lo[b, s] = first
            hi[b, s] = max(s + 1, min(end, x + p - b * S)) if causal else end
    return lo, hi


def attended(B, Sq, Sk, causal, q_start=None, key_lo=None, key_hi=None):
    """[B, Sq, Sk] truth values, and the positions [B, Sq] of the queries."""
    k = torch.arange(Sk)
    start = torch.full((B,), Sk - Sq) if q_start is None else q_start.long()
    pos = start[:, None] + torch.arange(Sq)
    m = torch.ones((B, Sq, Sk), dtype=torch.bool)
    if causal:
        m &= k <= pos[:, :, None]
    if key_lo is not None:
        m &= (k >= key_lo.long()[:, :, None]) & (k < key_hi.long()[:, :, None])
    return m, pos


def attention(Q, K, V, dO, scale, causal, cap=0.0, slopes=None, q_start=None, key_lo=None, key_hi=None):
    """O, LSE, dQ, dK, dV.  What a pair that is not attended holds takes no part."""
    B, Hq, Sq, D = Q.shape
    Hkv, Sk = K.shape[1:3]
    seen, pos = attended(B, Sq, Sk, causal, q_start, key_lo, key_hi)
    O, dQ = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape, dtype=torch.float64)
    dK, dV = torch.zeros(K.shape, dtype=torch.float64), torch.zeros(K.shape, dtype=torch.float64)
    LSE = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64)
    for b in range(B):
        rows, cols = seen[b].any(1), seen[b].any(0)
        if not rows.any():
            continue
        m = seen[b][rows][:, cols]
        far = (pos[b][rows][:, None] - torch.arange(Sk)[cols]).abs().double()
        for h in range(Hq):
            g = h // (Hq // Hkv)
            q, k, v, do = Q[b, h][rows].double(), K[b, g][cols].double(), V[b, g][cols].double(), dO[b, h][rows].double()
            z = q @ k.t() * scale
            gain = torch.full_like(z, scale)
            if cap:
                gain = gain * (1 - torch.tanh(z / cap) ** 2)
                z = cap * torch.tanh(z / cap)
            if slopes is not None:
                z = z - float(slopes[h]) * far
            z = z.masked_fill(~m, -math.inf)
            lse = torch.logsumexp(z, -1)
            P = torch.exp(z - lse[:, None])
            o = P @ v
            dP = do @ v.t()
            dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * gain      # (exactly zero where a query has one key)
            O[b, h, rows], LSE[b, h, rows], dQ[b, h, rows] = o, lse, dS @ k
            dK[b, g, cols] += dS.t() @ q
            dV[b, g, cols] += P.t() @ do
    return O, LSE, dQ, dK, dV
