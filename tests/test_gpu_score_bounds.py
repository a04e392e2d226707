"""Attention with rules on its scores at the ends of what its arguments may be."""
import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (lx: a fixture)
from util import FRO, rel_err_fro

pytestmark = pytest.mark.gpu


def test_more_pairs_than_a_launch_has_workgroups(lx):  # noqa: F811
    """2^23 sequences and heads, one query each, over the same 65 keys."""
    B, H, D, Sk = 1 << 15, 1 << 8, 64, 65
    g = torch.Generator(device="cuda").manual_seed(1)
    Q = torch.randn((B, H, 1, D), generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn((1, 1, Sk, D), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    O, LSE = torch.full_like(Q, float("nan")), torch.full((B, H, 1), float("nan"), device="cuda")
    lx.lx_score_attn_fwd(Q, k.expand(B, H, -1, -1), v.expand(B, H, -1, -1), 0.125, True, O, LSE)
    Q, O, LSE = Q.view(-1, D), O.view(-1, D), LSE.view(-1)
    for i in range(0, B * H, 1 << 20):
        z = torch.matmul(Q[i:i + (1 << 20)].float(), k[0, 0].float().t().contiguous()) * 0.125
        want = torch.matmul(torch.softmax(z, -1), v[0, 0].float())
        assert float((O[i:i + (1 << 20)].float() - want).norm() / want.norm()) <= FRO["bf16"]
        assert float((LSE[i:i + (1 << 20)] - torch.logsumexp(z, -1)).abs().max()) < 1e-4


CAPS = [128.0, 129.0, 1e3, 1e4, 1e6, 1e8, 3e38]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_large_caps(lx, cap, D):  # noqa: F811
    """A cap far above the scores changes nothing: O, LSE and the gradients within the gates of ordinary ones."""
    i = CAPS.index(cap)
    Call(lx, 1, 4, 2, 150, 150, D, ("f16", "bf16")[i % 2], seed=30 + i, cap=cap, slopes=i % 3 == 0).check()


@pytest.mark.parametrize("size", [(3, 8, 2, 1, 700), (1, 8, 2, 2, 4000), (1, 2, 2, 40, 300)], ids=str)      # whole pairs, equal runs, rows
@pytest.mark.parametrize("cap", [1e4, 1e7])
def test_large_caps_over_a_cache(lx, cap, size):  # noqa: F811
    Call(lx, *size, 64, "f16", seed=40, cap=cap).check(backward=False)


@pytest.mark.parametrize("size", [(1, 2, 1, 150, 150), (2, 4, 2, 1, 900)], ids=str)
@pytest.mark.parametrize("cap", [129.0, 400.0])
def test_scores_beyond_a_large_cap(lx, cap, size):  # noqa: F811
    """Scores of up to several caps.  Their fp32 arithmetic leaves a few 2^-24 of the cap: LSE 2^-21 of it, less than the gate of O by far."""
    c = Call(lx, *size, 64, "f16", seed=41, cap=cap)
    c.scale = 16.0
    c.forward()
    got, want = c.outputs()[:2], c.reference()[:2]
    assert rel_err_fro(got[0].numpy(), want[0].numpy()) <= FRO["f16"]
    assert float((got[1] - want[1]).abs().max()) <= cap * 2.0 ** -21


@pytest.mark.parametrize("size", [(1, 2, 1, 90, 90), (2, 4, 2, 1, 900)], ids=str)
@pytest.mark.parametrize("cap", [1e-3, 1e-20, 1e-38, 1e-42])
def test_small_caps(lx, cap, size):  # noqa: F811
    """Scores of nothing but the cap, a row of zeros among the queries."""
    c = Call(lx, *size, 64, "bf16", seed=42, cap=cap)
    c.Q[0, 0, 0] = 0
    c.check(backward=False)


@pytest.mark.parametrize("size", [(1, 2, 1, 150, 150), (2, 4, 2, 1, 900), (1, 2, 2, 1, 3000)], ids=str)      # rows, whole pairs, equal runs
@pytest.mark.parametrize("scale", [1e-18, 1e-25, 1e-38, 1e-42])
def test_scales_near_zero(lx, scale, size):  # noqa: F811
    """The bias by distance alone is left of the scores."""
    c = Call(lx, *size, 64, "bf16", seed=43, slopes=True)
    c.scale = scale
    c.check(backward=False)
    if size[3] > 1:
        c.backward()
        got, want = c.outputs(), c.reference()
        assert all(torch.isfinite(t).all() for t in got[2:])
        assert rel_err_fro(got[4].numpy(), want[4].numpy()) <= FRO["bf16"]


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "f16"), (128, "f16")])
@pytest.mark.parametrize("size", [(8, 32, 8, 1, 700), (2, 16, 4, 4, 3000)], ids=str)      # whole pairs, equal runs
def test_one_rounding_over_a_cache(lx, size, D, dtype):  # noqa: F811
    """P is not rounded to the element type: O is off by its own rounding alone, 2^-7 / sqrt(12) over a root mean square of 1.37 to 1.48 in a
    binade for bf16, 1.65e-3 at most, and a hundredth of it by chance."""
    c = Call(lx, *size, D, dtype, seed=44)
    c.forward()
    err = rel_err_fro(c.outputs()[0].numpy(), c.reference()[0].numpy())
    print(f"  O: fro {err:.3e}", flush=True)
    assert err <= (1.7e-3 if dtype == "bf16" else 1.7e-3 / 8)
