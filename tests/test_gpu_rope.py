"""Rotary positions (lx_rope, lx_rope_table) against the definition in 64 bits."""
import math

import pytest
import torch

import step_reference as ref
from util import torch_dtype

pytestmark = pytest.mark.gpu

# one rounding of the output, of at most half a unit in the last place, and three of fp32 before it
EPS = {"f32": 2.0 ** -22, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def near(got, want, dtype, size):
    """size: the largest |x| + |y| of a pair, which bounds the error of a cancelling sum."""
    assert torch.isfinite(got).all()
    err = (got.double().cpu() - want).abs()
    assert bool((err <= EPS[dtype] * want.abs() + 2.0 ** -22 * size).all()), float(err.max())


CASES = [  # B, S, Hq, Hkv, D, rot, layout
    (1, 1, 1, 1, 64, 64, "bshd"), (3, 1, 32, 8, 128, 128, "bhsd"), (2, 37, 5, 1, 64, 32, "bshd"), (1, 130, 3, 3, 80, 80, "bshd"),
    (2, 65, 4, 2, 96, 48, "bhsd"), (1, 51, 2, 1, 128, 118, "bshd"), (1, 40, 2, 2, 64, 2, "apart"), (1, 33, 2, 1, 65, 6, "odd"),
    (2, 300, 8, 8, 256, 256, "bshd")]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_turns(lx, case, dtype, interleaved):
    B, S, Hq, Hkv, D, rot, layout = case
    g = torch.Generator().manual_seed(7)

    def tensor(H):
        shape, cut = (B, S, H, D), 0
        if layout == "bhsd":
            t = torch.randn((B, H, S, D), generator=g)
        elif layout in ("apart", "odd"):      # every token's heads inside longer rows, from an odd element on
            cut = 8 if layout == "apart" else 3
            t = torch.randn((B, S, H, D + 2 * cut), generator=g).transpose(1, 2)
        else:
            t = torch.randn(shape, generator=g).transpose(1, 2)
        d = torch.empty_strided(t.shape, t.stride(), dtype=torch_dtype(dtype), device="cuda")
        d.copy_(t)
        return d[..., cut:cut + D]
    Q, K = tensor(Hq), tensor(Hkv)
    table = lx.lx_rope_table(rot, 500)
    pos = torch.randint(0, 500, (B, S), generator=g, dtype=torch.int32)
    Qo, Ko = torch.full_like(Q, math.nan), torch.full_like(K, math.nan)
    size = float(max(Q.abs().max(), K.abs().max())) * 2
    for inverse in (False, True):
        lx.lx_rope(Q, K, table, pos.cuda(), Qo, Ko, interleaved=interleaved, inverse=inverse)
        for x, y in ((Q, Qo), (K, Ko)):
            near(y, ref.rope(x.cpu(), table.cpu(), pos, interleaved, inverse), dtype, size)
            assert torch.equal(y[..., rot:], x[..., rot:])
    # in place, one tensor alone, positions by the token's number
    at = torch.arange(S, dtype=torch.int32).expand(B, S)
    want = ref.rope(Q.cpu(), table.cpu(), at, interleaved, False)
    lx.lx_rope(Q, None, table, None, Q, None, interleaved=interleaved)
    near(Q, want, dtype, size)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_backward_pass_is_the_transpose(lx, dtype):
    """<R x, y> = <x, R^T y>; in fp32 R^T R x = x, and differences along a direction."""
    g = torch.Generator().manual_seed(1)
    x, y = (torch.randn((2, 3, 50, 64), generator=g).to(torch_dtype(dtype)).cuda() for _ in range(2))
    table = lx.lx_rope_table(48, 64)
    Rx, Ry = torch.empty_like(x), torch.empty_like(y)
    lx.lx_rope(x, None, table, None, Rx, None, interleaved=True)
    lx.lx_rope(y, None, table, None, Ry, None, interleaved=True, inverse=True)
    a, b = float((Rx.double() * y.double()).sum()), float((x.double() * Ry.double()).sum())
    assert abs(a - b) <= 4 * EPS[dtype] * float(x.double().norm() * y.double().norm())
    if dtype == "f32":
        back = torch.empty_like(x)
        lx.lx_rope(Rx, None, table, None, back, None, interleaved=True, inverse=True)
        assert float((back - x).abs().max()) < 1e-6 * 8


@pytest.mark.parametrize("kind,kw", [(0, {}), (1, {"factor": 4.0}), (2, {"factor": 8.0}),
                                     (3, {"factor": 8.0, "trained_length": 8192.0, "low_turns": 1.0, "high_turns": 4.0, "gain": 1.2})])
def test_table(lx, kind, kw):
    rot, n, base = 48, 200001, 500000.0
    t = lx.lx_rope_table(rot, n, base, kind=kind, **kw).double().cpu()
    f = ref.rope_frequencies(rot, base, kind, kw.get("factor", 1.0), kw.get("trained_length", 0.0), kw.get("low_turns", 1.0), kw.get("high_turns", 32.0))
    angle = torch.arange(n, dtype=torch.float64)[:, None] * torch.tensor(f, dtype=torch.float64)
    gain = float(torch.tensor(kw.get("gain", 1.0), dtype=torch.float32))
    want = gain * torch.cat([angle.cos(), angle.sin()], 1)
    # rounded once to fp32 (factors are handed over in fp32); angles of 2e5 turns are known to 1e-10
    assert float((t - want).abs().max()) < 2.0 ** -23


def test_positions_outside_the_table(lx):
    x = torch.ones((1, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    lx.lx_rope(x, None, lx.lx_rope_table(32, 10), torch.tensor([[0, -1, 9, 10]], dtype=torch.int32, device="cuda"), out, None)
    assert torch.isnan(out[0, :, [1, 3], :32]).all() and torch.isfinite(out[0, :, [0, 2]]).all() and (out[..., 32:] == 1).all()


def test_offsets_beyond_32_bits(lx):
    room = torch.empty((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((2, 2, 3, 64), (1 << 32, 1024, 128, 1))
    y = torch.randn((2, 2, 3, 64)).bfloat16().cuda()
    x.copy_(y)
    table = lx.lx_rope_table(64, 8)
    out = torch.empty_like(y)
    lx.lx_rope(y, None, table, None, out, None)
    lx.lx_rope(x, None, table, None, x, None)
    assert torch.equal(x, out)


def test_refusals(lx):
    x = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
    table = lx.lx_rope_table(64, 10)
    for a, error in (((x, None, lx.lx_rope_table(66, 10), None, x, None), lx.LxError), ((x, None, table[:3], None, x, None), lx.LxError),
                     ((x, x.float(), table, None, x, x), AssertionError), ((x, None, table.half(), None, x, None), AssertionError),
                     ((x, None, table, torch.zeros((1, 4), device="cuda"), x, None), AssertionError),
                     ((x, None, table, torch.zeros((1, 5), dtype=torch.int32, device="cuda"), x, None), AssertionError),
                     ((x, None, table, None, x[:, :1].expand(-1, 2, -1, -1), None), lx.LxError),
                     ((x.double(), None, table, None, x.double(), None), lx.LxError)):
        with pytest.raises(error):
            lx.lx_rope(*a)
    for kw in ({"kind": 7}, {"kind": 1, "factor": 0.0}, {"kind": 3, "factor": 2.0}, {"base": -1.0}, {"gain": math.inf}):
        with pytest.raises(lx.LxError):
            lx.lx_rope_table(64, 10, **kw)
    with pytest.raises(lx.LxError):
        lx.lx_rope_table(2, 10, kind=2, factor=2.0)
    with pytest.raises(lx.LxError):
        lx.lx_rope_table(7, 10)
