"""Gradients where few of many keys carry a query's weight (steep slopes, large scores, a key that draws all queries), and where values have
a mean that their sum over the keys keeps: dP less its mean is then small against dP, and a mean from the rounded output shows.

Bounds, in squares of the rounding of numbers of all sizes, 1.67e-3 of a norm for bf16 (2^-9 / sqrt(3) times what the mean over a binade
adds): one for the result, one for dS, and for the mean at most four where it is not corrected:
sqrt(1 + 1 + 4) 1.67e-3 = 4.1e-3, an eighth of it for f16.  Where keys have a mean too the errors of dS add up along it: the gates."""
import math

import pytest
import torch

from score_centred import gradients
from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)
from util import FRO, rel_err_fro

pytestmark = pytest.mark.gpu
BOUND = {"bf16": 4.1e-3, "f16": 4.1e-3 / 8}


def check(c, bound, want=None):
    c.forward().backward()
    torch.cuda.synchronize()
    for name, x, y in zip(("dQ", "dK", "dV"), c.outputs()[2:], want or c.reference()[2:]):
        assert torch.isfinite(x).all(), name
        err = rel_err_fro(x.numpy(), y.numpy())
        print(f"  {name}: fro {err:.2e}", flush=True)
        assert err <= bound, (name, err)


def with_slope(c, slope):
    c.rules["slopes"] = torch.full((c.Q.shape[1],), slope, device="cuda")
    return c


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "f16"), (128, "f16")])
@pytest.mark.parametrize("slope", [0.25, 1.0, 2.0, 4.0])
def test_steep_slopes(lx, slope, D, dtype):  # noqa: F811
    check(with_slope(Call(lx, 1, 4, 2, 512, 512, D, dtype, seed=50), slope), BOUND[dtype])


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "f16")])
@pytest.mark.parametrize("size,cap", [(3.0, 0.0), (8.0, 0.0), (16.0, 0.0), (8.0, 50.0), (16.0, 400.0)])
def test_large_scores(lx, size, cap, D, dtype):  # noqa: F811
    """Scores of deviation `size`."""
    c = Call(lx, 1, 4, 2, 600, 600, D, dtype, seed=51, cap=cap)
    c.Q.mul_(size / (2.0 if cap else 1.0))
    check(c, BOUND[dtype])


@pytest.mark.parametrize("B", [1, 40])          # two teams of wavefronts, one
@pytest.mark.parametrize("D", [64, 128])
def test_all_kinds_of_heads(lx, D, B):  # noqa: F811
    """Heads that attend broadly next to steep ones, and a key that draws the queries of one batch entry."""
    c = Call(lx, B, 4, 4, 520, 520, D, "bf16", seed=52)
    c.rules["slopes"] = torch.tensor([0.0, 0.01, 1.0, 3.0], device="cuda")
    c.Q[0] += 8 * math.sqrt(D) * c.K[0, :, :1] / c.K[0, :, :1].float().square().sum(-1, keepdim=True).to(c.K.dtype)
    check(c, BOUND["bf16"])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("means", [(1.0, 0.0), (3.0, 0.0), (1.0, 1.0), (0.1, 1.0)])      # of values, of keys
def test_means(lx, means, dtype):  # noqa: F811
    c = Call(lx, 1, 4, 4, 1024, 1024, 64, dtype, seed=53)
    g = torch.Generator(device="cuda").manual_seed(1)
    for t, m in zip((c.V, c.K), means):
        t += m * torch.randn((1, 4, 1, 64), generator=g, device="cuda").to(t.dtype)
    check(c, FRO[dtype])


@pytest.mark.parametrize("B", [1, 20])
def test_masked_places_that_are_not_finite(lx, B):  # noqa: F811
    """Both reasons for another pass in the same workgroups: steep slopes, and NaN behind the documents' ends."""
    S = 700
    lo, hi = torch.zeros((B, S), dtype=torch.int64), (torch.arange(S) + 1).expand(B, S).clone()
    lo[:, 300:], lo[:, 330:] = 300, 330
    lo[:, 300:330] = hi[:, 300:330] = 0
    c = with_slope(Call(lx, B, 4, 2, S, S, 64, "bf16", seed=54, causal=False, key_lo=lo, key_hi=hi), 2.0)
    for t, value in ((c.K, math.nan), (c.V, math.inf), (c.Q, -math.inf), (c.dO, math.nan)):
        t[:, :, 300:330] = value
    check(c, BOUND["bf16"])


def test_same_bits(lx):  # noqa: F811
    got = []
    for _ in range(2):
        c = with_slope(Call(lx, 1, 4, 2, 600, 600, 128, "bf16", seed=56), 1.0).forward().backward()
        got.append([t.clone() for t in (c.dQ, c.dK, c.dV)])
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("size", [(1, 1, 1, 2, 2), (1, 2, 1, 60, 60), (2, 2, 2, 7, 100)], ids=str)
@pytest.mark.parametrize("scores", [2.0, 6.0, 12.0])
def test_single_precision(lx, size, scores):  # noqa: F811
    """The correctness configuration: sums in 64 bits, the mean of dP and the softmax's sum among them, so that dQ, dK and dV carry one
    rounding, 2^-24 of an element at most; as much again for all else."""
    for seed in range(4):
        c = Call(lx, *size, 64, "f32", seed=90 + seed, slopes=seed == 3)
        c.Q.mul_(scores)
        slopes = c.rules["slopes"]
        check(c, 2.0 ** -23, gradients(*(t.cpu() for t in (c.Q, c.K, c.V, c.dO)), c.scale, True, None if slopes is None else slopes.cpu()))
