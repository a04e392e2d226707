"""The gradients in 64 bits that the peaked single-precision tests are held against: against the formula of two keys, in which nothing cancels,
and against the plain definition where that has all its digits."""
import math

import pytest
import torch

import step_reference
from score_centred import gradients


def inputs(B, Hq, Hkv, Sq, Sk, size, seed):
    g = torch.Generator().manual_seed(seed)
    Q, K, V, dO = (torch.randn((B, H, S, 64), generator=g) for H, S in ((Hq, Sq), (Hkv, Sk), (Hkv, Sk), (Hq, Sq)))
    return Q * size, K, V, dO


@pytest.mark.parametrize("size", [1.0, 6.0, 12.0, 30.0])
@pytest.mark.parametrize("seed", range(4))
def test_two_keys(size, seed):
    """dS of keys 0 and 1 is +-p0 p1 (dP0 - dP1).  A score's error, 1e-15 of the sum of its products' sizes (below 1e3), is P's relative one:
    1e-12; the difference of dP loses a digit or two of its 16."""
    Q, K, V, dO = inputs(1, 1, 1, 1, 2, size, seed)
    q, k, v, d = (t[0, 0].double() for t in (Q, K, V, dO))
    z, dP = k @ q[0] / 8, v @ d[0]
    gap = float(z[1] - z[0])
    ds = float(dP[0] - dP[1]) / ((1 + math.exp(gap)) * (1 + math.exp(-gap))) / 8
    dQ, dK, _ = gradients(Q, K, V, dO, 0.125, False)
    for got, want in ((dQ[0, 0, 0], ds * (k[0] - k[1])), (dK[0, 0], torch.stack((ds * q[0], -ds * q[0])))):
        assert (got - want).norm() <= 1e-11 * want.norm()


@pytest.mark.parametrize("causal,slopes", [(True, None), (False, torch.tensor([0.0, 0.1, 0.2, 0.3]))])
def test_broad_weights(causal, slopes):
    x = inputs(2, 4, 2, 9, 30, 1.0, 7)
    for got, want in zip(gradients(*x, 0.125, causal, slopes), step_reference.attention(*x, 0.125, causal, slopes=slopes)[2:]):
        assert (got - want).norm() <= 1e-12 * want.norm()
