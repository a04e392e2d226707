"""Attention of a few queries per sequence over a cache, its keys split among wavefronts and joined."""
import math

import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (lx: a fixture)
from util import FRO, rel_err_fro

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, Sq, C: one sequence and head; more parts than wavefronts ever join at once; more than 64 sequences; more rows of a key
# head than one tile holds; lengths of one, none, a tile and one more
CASES = [(1, 1, 1, 1, 65, [65]), (1, 1, 1, 1, 9000, [9000]), (2, 8, 2, 1, 700, [700, 1]), (3, 4, 4, 2, 333, [333, 0, 34]),
         (70, 2, 1, 1, 200, [(37 * i) % 201 for i in range(70)]), (2, 64, 1, 1, 500, [500, 77]), (2, 8, 1, 5, 400, [400, 129]),
         (5, 2, 2, 3, 1000, [0, 1000, 0, 32, 0]), (130, 1, 1, 1, 70, [0] * 129 + [70]), (1, 2, 1, 16, 129, [128])]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c[:5]))
def test_lengths(lx, case, D):
    B, Hq, Hkv, Sq, C, lengths = case
    i = CASES.index(case)
    c = Call(lx, B, Hq, Hkv, Sq, C, D, ("bf16", "f16")[(i + D // 64) % 2], ("bshd", "bhsd", "apart")[i % 3], seed=20 + i,
             cap=(0.0, 5.0)[i // 2 % 2], slopes=i % 2 == 0, q_start=torch.tensor(lengths) - Sq)
    # what a cache holds behind a sequence's end
    for b, n in enumerate(lengths):
        for t in (c.K, c.V):
            t[b, :, n:] = (math.nan, math.inf, -math.inf)[b % 3]
    c.check(backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_intervals(lx, dtype):
    """Windows of a cache, some empty: from the middle of a tile to the middle of another."""
    lo, hi = torch.tensor([[5, 0], [700, 100], [0, 0], [333, 334]]), torch.tensor([[600, 3], [1000, 900], [0, 0], [334, 1000]])
    Call(lx, 4, 4, 2, 2, 1000, 64, dtype, seed=41, causal=False, slopes=True, key_lo=lo, key_hi=hi,
         q_start=torch.tensor([998, 998, 998, 0])).check(backward=False)


def test_not_finite_in_an_attended_row(lx):
    c = Call(lx, 2, 2, 1, 1, 500, 64, "bf16", seed=42, q_start=torch.tensor([499, 299]))
    c.V[:, 0, 299, 5] = math.nan
    c.V[:, 0, 498, 6] = math.inf
    c.forward()
    assert torch.isnan(c.O[:, :, 0, 5]).all() and torch.isfinite(c.LSE).all()
    assert not torch.isfinite(c.O[0, :, 0, 6]).any()


def test_cache_of_more_than_32_bits(lx):
    """A token every 2^22 elements: the last ones lie beyond 2^32 bytes, and beyond 2^32 elements."""
    c = Call(lx, 1, 2, 1, 1, 1100, 64, "bf16", seed=43)
    room = torch.empty(1100 << 22, dtype=torch.bfloat16, device="cuda")
    for i, name in enumerate(("K", "V")):
        far = room[64 * i:].as_strided((1, 1, 1100, 64), (1 << 30, 64, 1 << 22, 1))
        far.copy_(getattr(c, name))
        setattr(c, name, far)
    c.check(backward=False)


def test_same_as_by_rows(lx):
    """The same queries as the last ones of a longer call, whose keys are not split."""
    a = Call(lx, 2, 4, 2, 128, 700, 64, "f16", seed=44, slopes=True)
    a.forward()
    O = torch.empty_like(a.O[:, :, -3:])
    lx.lx_score_attn_fwd(a.Q[:, :, -3:], a.K, a.V, a.scale, True, O, None, slopes=a.rules["slopes"])
    assert rel_err_fro(O.double().cpu().numpy(), a.O[:, :, -3:].double().cpu().numpy()) <= FRO["f16"]


def test_same_bits_twice(lx):
    got = []
    for _ in range(2):
        c = Call(lx, 3, 8, 2, 1, 5000, 128, "bf16", seed=45, cap=5.0, q_start=torch.tensor([4999, 17, 3000]))
        got.append(c.forward().O.clone())
    assert torch.equal(*got)
