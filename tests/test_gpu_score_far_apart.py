"""Gradients of queries with few keys that lie far apart: only the tiles that they attend are read for their Delta."""
import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)
from test_gpu_score_few_keys import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_short_intervals_far_apart(lx, D):  # noqa: F811
    """1 to 32 keys anywhere among 3000, some queries with none."""
    g = torch.Generator().manual_seed(2)
    lo = torch.randint(0, 2990, (2, 300), generator=g)
    hi = lo + torch.randint(0, 33, (2, 300), generator=g)
    check(Call(lx, 2, 4, 2, 300, 3000, D, "bf16", seed=55, causal=False, key_lo=lo, key_hi=hi))

