"""The gradients of attention in 64 bits where one key has nearly all of a query's weight.

dP less its mean under P is then as small against dP as the other keys' weight: the mean itself, in 64 bits, leaves one digit at a weight of
1e-15 and none below.  Here dP is taken less that of the query's heaviest key first, so that no digits cancel."""
import math

import torch

from step_reference import attended


def gradients(Q, K, V, dO, scale, causal, slopes=None):
    """dQ, dK, dV of queries that all attend a key (no cap)."""
    B, Hq, Sq, _ = Q.shape
    Hkv, Sk = K.shape[1:3]
    seen, pos = attended(B, Sq, Sk, causal)
    Q, K, V, dO = (t.double() for t in (Q, K, V, dO))
    dQ, dK, dV = torch.zeros_like(Q), torch.zeros_like(K), torch.zeros_like(V)
    for b in range(B):
        far = (pos[b][:, None] - torch.arange(Sk)).abs().double()
        for h in range(Hq):
            g = h // (Hq // Hkv)
            z = Q[b, h] @ K[b, g].t() * scale
            if slopes is not None:
                z = z - float(slopes[h]) * far
            z = z.masked_fill(~seen[b], -math.inf)
            top, at = z.max(-1, keepdim=True)
            w = torch.exp(z - top)
            P = w / w.sum(-1, keepdim=True)
            dP = dO[b, h] @ V[b, g].t()
            dP = dP - dP.gather(-1, at)
            dS = P * (dP - (P * dP).sum(-1, keepdim=True)) * scale
            dQ[b, h] = dS @ K[b, g]
            dK[b, g] += dS.t() @ Q[b, h]
            dV[b, g] += P.t() @ dO[b, h]
    return dQ, dK, dV
