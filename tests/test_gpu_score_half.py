"""Half precision ends at 65504 and gets coarse below 2^-14: gradients far below and above one, weights of many keys.  The same gates as for
numbers of order one (a result that itself lies below 2^-14 has half a unit of 2^-24 instead: sizes here keep results above)."""
import math

import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)
from util import FRO, rel_err_fro

pytestmark = pytest.mark.gpu


def check(c, names=("O", "LSE", "dQ", "dK", "dV")):
    c.forward().backward()
    torch.cuda.synchronize()
    for name, x, y in zip(("O", "LSE", "dQ", "dK", "dV"), c.outputs(), c.reference()):
        if name == "LSE" or name not in names:
            continue
        assert torch.isfinite(x).all(), name
        err = rel_err_fro(x.numpy(), y.numpy())
        print(f"  {name}: fro {err:.2e}", flush=True)
        assert err <= FRO["f16"], (name, err)


@pytest.mark.parametrize("size", [(1, 2, 1, 1500, 1500, 64), (1, 2, 2, 700, 700, 128), (9, 8, 8, 600, 600, 64)], ids=str)      # one and two teams
@pytest.mark.parametrize("dO", [1e-3, 1.0, 300.0])
def test_small_and_large_gradients(lx, size, dO):  # noqa: F811
    """Scores are scaled so that dQ and dK, of the order of dO scale / sqrt(keys), are representable: by 16 where dO is small."""
    c = Call(lx, *size, "f16", seed=60, cap=(0.0, 5.0)[size[0] > 1])
    c.Q.mul_(2.0 ** -7 if dO < 1 else 1.0)
    c.scale = 16.0 if dO < 1 else c.scale
    c.dO.mul_(dO)
    check(c)


@pytest.mark.parametrize("D", [64, 128])
def test_gradients_of_many_sizes(lx, D):  # noqa: F811
    """A factor of 2^24 between the gradients of some queries and others: each row of dQ as exact as its neighbours'.  Elements that are
    beyond half precision themselves, in the last rows, are infinite."""
    c = Call(lx, 1, 2, 2, 400, 400, D, "f16", seed=61)
    c.scale = 4.0
    c.Q.mul_(2.0 ** -5)
    c.dO *= (2.0 ** (torch.arange(400, device="cuda") % 25 - 12))[:, None].half()
    check(c, ("dK", "dV"))
    got, want = c.dQ.double().cpu(), c.reference()[2]
    for e in range(10, 25):       # rows of 2^-2 and more: above 2^-14 in all but few elements
        x, y = got[:, :, e::25], want[:, :, e::25]
        beyond = y.abs() >= 65504 * (1 + FRO["f16"])
        assert torch.isinf(x[beyond]).all()
        held = torch.isfinite(x)
        assert (y[~held].abs() >= 65504 * (1 - 4 * FRO["f16"])).all()
        assert rel_err_fro(x[held].numpy(), y[held].numpy()) <= FRO["f16"], e


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_products_beyond_the_range(lx, D, causal):  # noqa: F811
    """dO and V so large that dS passes 65504, and a scale that brings dQ and dK back."""
    c = Call(lx, 2, 2, 1, 90, 90, D, "f16", seed=62, causal=causal)
    c.scale = 2.0 ** -10
    c.dO.mul_(256.0)
    c.V.mul_(512.0)
    check(c, ("O", "dQ", "dK", "dV"))


@pytest.mark.parametrize("S", [40, 700])
@pytest.mark.parametrize("mean", [0.0, 1.0])
def test_small_values(lx, S, mean):  # noqa: F811
    """V below 2^-14, where half precision is coarse: O is 2^-25 off whatever its size, and Delta from it as much more."""
    c = Call(lx, 1, 2, 1, S, S, 64, "f16", seed=66)
    c.V.mul_(2.0 ** -16)
    c.K += mean
    c.dO.mul_(1024.0)
    c.scale = 2.0
    c.Q.mul_(2.0 ** -4)
    check(c, ("dQ", "dK", "dV"))


def test_large_values_of_one_key(lx):  # noqa: F811
    """A row of V of thousands among ordinary ones: the query side makes room for it, other rows stay as they are."""
    c = Call(lx, 1, 2, 2, 300, 300, 64, "f16", seed=63)
    c.scale = 2.0 ** -6
    c.V[:, :, 150] *= 8192.0
    check(c, ("O", "dQ", "dK", "dV"))


@pytest.mark.parametrize("Sk", [20000, 131072])
def test_weights_of_many_keys(lx, Sk):  # noqa: F811
    """P of 1 / Sk lies among the numbers that half precision holds coarsely.  (dO of 32: dV, dO sqrt(Sq) / Sk, is held well.)"""
    c = Call(lx, 1, 2, 1, 40, Sk, 64, "f16", seed=64, causal=False)
    c.dO.mul_(1024.0)
    c.scale = 1.0
    c.Q.mul_(0.125)
    check(c, ("dQ", "dK", "dV"))


@pytest.mark.parametrize("value", [math.nan, math.inf, 60000.0])
def test_masked_gradients_take_no_part(lx, value):  # noqa: F811
    """Padding queries whose dO is not finite, or enormous, beside queries with small gradients."""
    S = 300
    lo, hi = torch.zeros((1, S), dtype=torch.int64), (torch.arange(S) + 1)[None].clone()
    lo[0, 200:] = hi[0, 200:] = 0
    c = Call(lx, 1, 2, 1, S, S, 64, "f16", seed=65, causal=False, key_lo=lo, key_hi=hi)
    c.Q.mul_(2.0 ** -7)
    c.scale = 16.0
    c.dO.mul_(1e-3)
    c.dO[:, :, 200:] = value
    c.Q[:, :, 200:] = value
    check(c)


@pytest.mark.parametrize("seed", range(275, 279))
def test_small_gradients_of_few_queries(lx, seed):  # noqa: F811
    """Where few queries attend and the scores are large, most P are far below one: a bound of dS that is 2^-8 of the keys' number is not
    yet one at which dS is coarse, its parts are."""
    c = Call(lx, 1, 4, 4, 21, 212, 64, "f16", seed=seed, cap=8.0)
    c.Q.mul_(6)
    c.dO.mul_(0.01)
    check(c)
