"""Attention over a cache where the keys of all pairs are one sequence that workgroups share out in equal runs: more than 64 and
more than 128 sequences, several tiles of rows, lengths from none up, runs of a unit, and whole pairs within a run."""
import math

import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, Sq, C, lengths
CASES = [(1, 1, 1, 1, 1025, [1025]), (70, 2, 1, 1, 1300, [(397 * i) % 1301 for i in range(70)]),
         (127, 1, 1, 1, 4200, [0] * 63 + [4200] + [1] * 62 + [129]), (3, 64, 1, 1, 1500, [1500, 0, 700]), (2, 16, 2, 5, 2100, [2100, 1027]),
         (1, 8, 8, 16, 5000, [4999]), (40, 3, 3, 2, 1100, [128 * (i % 9) + (i % 3) for i in range(40)]), (5, 2, 2, 1, 1200, [0] * 5)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c[:5]))
def test_parts(lx, case, D):  # noqa: F811
    B, Hq, Hkv, Sq, C, lengths = case
    i = CASES.index(case)
    dtype = ("bf16", "f16")[(i + D // 64) % 2]
    assert lx.lx_score_attn_fwd_workspace_bytes({"bf16": lx.LX_BF16, "f16": lx.LX_F16}[dtype], B, Hq, Hkv, Sq, C, D) > 0
    c = Call(lx, B, Hq, Hkv, Sq, C, D, dtype, ("bshd", "bhsd", "apart")[i % 3], seed=60 + i, cap=(0.0, 5.0)[i % 2], slopes=i % 3 == 0,
             q_start=torch.tensor(lengths) - Sq)
    for b, n in enumerate(lengths):       # behind a sequence's end
        for t in (c.K, c.V):
            t[b, :, n:] = (math.nan, math.inf, -math.inf)[b % 3]
    c.check(backward=False)


def test_windows(lx):  # noqa: F811
    """Windows that begin at any key, one of them beyond 1024 others."""
    lo = torch.tensor([[1999], [5], [0], [1200]])
    hi = torch.tensor([[2000], [1999], [0], [1460]])
    Call(lx, 4, 6, 2, 1, 2000, 128, "bf16", seed=71, causal=False, key_lo=lo, key_hi=hi).check(backward=False)
