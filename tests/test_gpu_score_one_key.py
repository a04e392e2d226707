"""Queries with a single key: O is its value, and no gradient reaches the query - exactly none, whatever the rules on the score.  Nor the
key: none at all from sequences of one token, and but the rounding of P to fp32 (2^-21 of dO V) where it stands among others."""
import math

import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (30.0, False), (5.0, True), (300.0, False)])
@pytest.mark.parametrize("B,D", [(1, 64), (1, 128), (300, 64), (300, 128)])       # two teams of wavefronts, one
def test_one_token(lx, B, D, cap, slopes, dtype):  # noqa: F811
    c = Call(lx, B, 8, 4, 1, 1, D, dtype, seed=80, causal=False, cap=cap, slopes=slopes).forward().backward()
    assert torch.equal(c.O, c.V.repeat_interleave(2, 1))
    assert not c.dQ.any() and not c.dK.any()
    want = c.dO.float().view(B, 4, 2, 1, D).sum(2)
    assert float((c.dV.float() - want).abs().max()) <= 2.0 ** -8 * float(want.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_among_others(lx, dtype):  # noqa: F811
    """Causal: the first query has one key.  Documents of one token here and there; all queries on the last key of a tile and one."""
    Call(lx, 2, 4, 2, 200, 200, 64, dtype, seed=81, cap=20.0).check()
    c = Call(lx, 2, 4, 2, 200, 200, 64, dtype, seed=81, cap=20.0).forward().backward()
    assert not c.dQ[:, :, 0].any()
    lo = torch.arange(200).expand(2, 200) // 3 * 3
    hi = torch.minimum(lo + torch.tensor([1, 3])[:, None], torch.tensor(200))
    c = Call(lx, 2, 4, 2, 200, 200, 64, dtype, seed=82, causal=False, cap=20.0, key_lo=lo, key_hi=hi).forward().backward()
    assert not c.dQ[0].any() and c.dQ[1].any() and float(c.dK[0].abs().max()) <= 2.0 ** -18 * float(c.dK[1].abs().max())
    lo = torch.full((1, 70), 128)
    c = Call(lx, 1, 2, 1, 70, 129, 64, dtype, seed=83, causal=False, cap=20.0, key_lo=lo, key_hi=lo + 1).forward().backward()
    assert not c.dQ.any() and not c.dK[:, :, :128].any() and not c.dV[:, :, :128].any() and c.dV[:, :, 128].any()
    assert float(c.dK.abs().max()) <= 1e-4 and torch.isfinite(c.dV).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_is_not_hidden(lx, dtype):  # noqa: F811
    c = Call(lx, 1, 1, 1, 1, 1, 64, dtype, seed=84, causal=False)
    c.dO[0, 0, 0, 3] = math.nan
    c.forward().backward()
    assert torch.isnan(c.dQ).all() and torch.isnan(c.dK).all() and torch.isnan(c.dV[0, 0, 0, 3])
