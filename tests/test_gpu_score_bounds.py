"""Attention with rules on its scores at the ends of what its arguments may be."""
import pytest
import torch

from test_gpu_score_attn import lx  # noqa: F401  (a fixture)
from util import FRO

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
