"""Key ranges that hold any numbers: below zero, past the keys, the lowest and the highest of their type, end before begin.  A
query whose interval holds no key gives zeros, and nothing outside the keys is read."""
import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


def extremes(B, Sq, Sk):
    pairs = [(0, LOW), (5, LOW), (Sk, HIGH), (HIGH, HIGH), (HIGH, LOW), (LOW, HIGH), (LOW, LOW), (-7, 9), (Sk - 3, HIGH), (40, 3), (3, 40),
             (Sk + 100, Sk + 200), (-200, -100)]
    t = torch.tensor([pairs[i * 7 % len(pairs)] for i in range(B * Sq)], dtype=torch.int64).view(B, Sq, 2)
    return t[..., 0].contiguous(), t[..., 1].contiguous()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Sk,D,dtype", [(2, 4, 2, 200, 333, 64, "bf16"), (1, 2, 1, 130, 130, 128, "f16"), (3, 2, 2, 40, 70, 64, "f32")])
def test_training(lx, B, Hq, Hkv, Sq, Sk, D, dtype, causal):  # noqa: F811
    lo, hi = extremes(B, Sq, Sk)
    Call(lx, B, Hq, Hkv, Sq, Sk, D, dtype, seed=Sk, causal=causal, slopes=True, cap=8.0, key_lo=lo, key_hi=hi).check()


@pytest.mark.parametrize("Sq,Sk", [(1, 700), (3, 5000), (7, 64)])
def test_few_queries(lx, Sq, Sk):  # noqa: F811
    lo, hi = extremes(13, Sq, Sk)
    Call(lx, 13, 4, 2, Sq, Sk, 128, "bf16", seed=Sq, causal=False, key_lo=lo, key_hi=hi).check(backward=False)


@pytest.mark.parametrize("Sq,Sk", [(96, 200), (1, 3000)])
def test_nobody_attends(lx, Sq, Sk):  # noqa: F811
    lo, hi = torch.full((2, Sq), 17), torch.full((2, Sq), LOW, dtype=torch.int64)
    c = Call(lx, 2, 4, 4, Sq, Sk, 64, "bf16", key_lo=lo, key_hi=hi)
    c.check()
    assert not any(t.any() for t in (c.O, c.dQ, c.dK, c.dV)) and torch.isinf(c.LSE).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,S", [(1, 260), (2, 4096)])       # two teams of wavefronts, one
def test_all_attend_the_same_keys(lx, B, S, D):  # noqa: F811
    """Every query attends keys 0 .. 99, and what lies behind them in the same tile is not finite."""
    c = Call(lx, B, 4, 2, S, 512, D, "bf16", seed=D, causal=False, key_lo=torch.zeros(B, S), key_hi=torch.full((B, S), 100))
    for i, t in enumerate((c.K, c.V)):
        t[:, :, 100:110] = float("nan")
        t[:, :, 110:] = float(("inf", "-inf")[i])
    c.check()
    assert not c.dK[:, :, 100:].any() and not c.dV[:, :, 100:].any()
