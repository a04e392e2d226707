"""Attention with rules on its scores (lx_score_attn_fwd / _bwd, lx_attn_key_ranges) against the definition in 64 bits."""
import math

import pytest
import torch

import step_reference as ref
from util import FRO, TOL, rel_err_fro, rel_err_max, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def tensor(g, B, H, S, D, dtype, layout="bshd", scale=1.0):
    """[B,H,S,D] on the device: "bhsd", "bshd" or "apart" (a slice of longer rows and heads)."""
    if layout == "bhsd":
        t = torch.randn((B, H, S, D), generator=g)
    elif layout == "bshd":
        t = torch.randn((B, S, H, D), generator=g).transpose(1, 2)
    else:
        t = torch.randn((B, S, H + 1, D + 24), generator=g).transpose(1, 2)[:, :H, :, 8:8 + D]
    # (a copy to the device keeps the strides of a dense tensor only: lay the slice out there)
    d = torch.empty_strided(t.shape, t.stride(), dtype=torch_dtype(dtype), device="cuda")
    d.copy_(t * scale)
    return d


class Call:
    """Inputs of a call and its outputs, filled with NaN before."""

    def __init__(self, lx, B, Hq, Hkv, Sq, Sk, D, dtype, layout="bshd", seed=0, causal=True, cap=0.0, slopes=False, **rules):
        g = torch.Generator().manual_seed(1000 + seed)
        self.lx, self.dtype, self.causal, self.scale = lx, dtype, causal, D ** -0.5
        self.Q = tensor(g, B, Hq, Sq, D, dtype, layout, 2.0 if cap else 1.0)
        self.K, self.V = tensor(g, B, Hkv, Sk, D, dtype, layout), tensor(g, B, Hkv, Sk, D, dtype, layout)
        self.dO = tensor(g, B, Hq, Sq, D, dtype, layout)
        self.O, self.dQ = (torch.full_like(self.Q, math.nan) for _ in range(2))
        self.dK, self.dV = (torch.full_like(self.K, math.nan) for _ in range(2))
        self.LSE = torch.full((B, Hq, Sq), math.nan, device="cuda")
        self.rules = {"cap": cap, "slopes": (torch.rand(Hq, generator=g) * 0.3).cuda() if slopes else None}
        self.rules.update({k: None if v is None else v.to(torch.int32).cuda() for k, v in rules.items()})

    def forward(self):
        self.lx.lx_score_attn_fwd(self.Q, self.K, self.V, self.scale, self.causal, self.O, self.LSE, **self.rules)
        return self

    def backward(self):
        self.lx.lx_score_attn_bwd(self.Q, self.K, self.V, self.O, self.LSE, self.dO, self.scale, self.causal, self.dQ, self.dK,
                                  self.dV, **self.rules)
        return self

    def outputs(self):
        return [t.double().cpu() for t in (self.O, self.LSE, self.dQ, self.dK, self.dV)]

    def reference(self):
        rules = {k: v.cpu() if torch.is_tensor(v) else v for k, v in self.rules.items()}
        return ref.attention(*(t.cpu() for t in (self.Q, self.K, self.V, self.dO)), self.scale, self.causal, **rules)

    def check(self, backward=True):
        """Two roundings to the element type on the way to an output (P or dS, and the output): the gates of tests/util.py.  LSE is
        fp32 throughout; a score is a sum of D products of 16-bit numbers, |error| <= D 2^-24 sum |q k| scale, below 1e-4 here."""
        self.forward()
        if backward:
            self.backward()
        torch.cuda.synchronize()
        got, want = self.outputs(), self.reference()
        for name, x, y in list(zip(("O", "LSE", "dQ", "dK", "dV"), got, want))[:5 if backward else 2]:
            if name == "LSE":
                none = torch.isinf(y)
                assert torch.equal(none, torch.isinf(x)) and not torch.isnan(x).any()
                assert (x[~none] - y[~none]).abs().max() < 1e-4 if (~none).any() else True
                continue
            assert torch.isfinite(x).all(), name
            top, fro = rel_err_max(x.numpy(), y.numpy()), rel_err_fro(x.numpy(), y.numpy())
            print(f"  {name}: max {top:.2e} fro {fro:.2e}", flush=True)
            assert top <= TOL[self.dtype] and fro <= FRO[self.dtype], (name, top, fro)


def ranges(kind, B, S, seed=0):
    """key_lo, key_hi of a self-attention: what lx_attn_key_ranges would not write."""
    g = torch.Generator().manual_seed(seed)
    q = torch.arange(S).expand(B, S)
    if kind == "any":              # in no order, some empty, some outside the keys
        lo = torch.randint(-5, S + 5, (B, S), generator=g)
        hi = lo + torch.randint(-3, S, (B, S), generator=g)
    elif kind == "none":
        lo, hi = torch.full((B, S), 3), torch.full((B, S), 3)
    elif kind == "one":            # one key each, the last rows none
        lo = (q * 7) % S
        hi = torch.where(q < S - S // 4, lo + 1, lo)
    else:                          # a window
        lo, hi = q - 17, q + 1
    return {"key_lo": lo, "key_hi": hi}


SIZES = [(1, 1, 1, 1, 1), (2, 2, 1, 1, 77), (1, 4, 2, 3, 3), (2, 3, 3, 63, 63), (1, 2, 2, 64, 64), (1, 4, 1, 65, 65), (1, 2, 2, 128, 128),
         (2, 6, 2, 129, 129), (1, 2, 1, 100, 333), (1, 2, 2, 333, 100), (1, 1, 1, 700, 700)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(lx, size, D):
    B, Hq, Hkv, Sq, Sk = size
    i = SIZES.index(size)
    # every type, layout, mask and rule over the sizes
    Call(lx, B, Hq, Hkv, Sq, Sk, D, ("bf16", "f16")[i % 2], ("bshd", "bhsd", "apart")[i % 3], seed=i, causal=i % 4 != 2,
         cap=(0.0, 5.0, 30.0)[i % 3], slopes=(i + D // 64) % 2 == 0).check()


@pytest.mark.parametrize("cap,slopes", [(0.0, False), (0.0, True), (4.0, False), (4.0, True)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rules(lx, dtype, D, cap, slopes):
    Call(lx, 1, 4, 2, 150, 150, D, dtype, seed=3, cap=cap, slopes=slopes).check()


@pytest.mark.parametrize("kind", ["any", "none", "one", "window"])
@pytest.mark.parametrize("dtype,D,S", [("bf16", 64, 200), ("f16", 128, 321), ("f32", 64, 70)])
def test_ranges(lx, kind, dtype, D, S):
    Call(lx, 2, 4, 2, S, S, D, dtype, seed=5, causal=False, slopes=True, **ranges(kind, 2, S, seed=S)).check()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 128), ("f32", 128)])
def test_positions_of_the_queries(lx, dtype, D):
    # before the first key (nothing attended), in the middle, behind the last
    Call(lx, 4, 2, 1, 5, 90, D, dtype, seed=6, slopes=True, q_start=torch.tensor([-9, -2, 40, 200])).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("causal,with_prefix", [(True, False), (True, True), (False, False)])
def test_packed_documents(lx, dtype, causal, with_prefix):
    B, S = 3, 150
    # a document over a row's end, one of a single token, gaps, an empty row's end
    docs = [(0, 1, 1), (1, 40, 7), (40, 64, 0), (70, 149, 100), (149, 200, 3), (210, 290, 20), (310, 400, 200)]
    begin, end, prefix = (torch.tensor(x, dtype=torch.int32).cuda() for x in zip(*docs))
    lo, hi = (torch.full((B, S), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    lx.lx_attn_key_ranges(begin, end, prefix if with_prefix else None, causal, lo, hi)
    want = ref.key_ranges(B, S, docs if with_prefix else [(x, y, 0) for x, y, _ in docs], causal)
    assert torch.equal(lo.cpu(), want[0]) and torch.equal(hi.cpu(), want[1])
    Call(lx, B, 2, 2, S, S, 64, dtype, seed=8, causal=False, slopes=True, key_lo=lo, key_hi=hi).check()


def test_no_documents(lx):
    lo, hi = (torch.full((2, 5), 9, dtype=torch.int32, device="cuda") for _ in range(2))
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    lx.lx_attn_key_ranges(none, none, None, True, lo, hi)
    assert int(lo.abs().sum()) == 0 and int(hi.abs().sum()) == 0


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f16", 64), ("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_masked_places_hold_anything(lx, dtype, D, value):
    """Padding queries, keys behind a sequence's end and other documents hold NaN or infinities: no other row notices."""
    S = 210
    lo, hi = torch.zeros((1, S), dtype=torch.int64), torch.arange(1, S + 1)[None].clone()
    lo[0, 70:], lo[0, 90:] = 70, 90
    hi[0, 90:] = hi[0, 90:].clamp(max=170)
    lo[0, 70:90] = hi[0, 70:90] = 0          # queries 70 .. 89 attend nothing
    hi[0, 170:] = 0
    c = Call(lx, 1, 2, 1, S, S, D, dtype, seed=9, causal=False, key_lo=lo, key_hi=hi)
    for t in (c.Q, c.dO):
        t[:, :, 70:90] = value
        t[:, :, 170:] = value
    for t in (c.K, c.V):
        t[:, :, 70:90] = value
        t[:, :, 170:] = value
    c.forward().backward()
    got, want = c.outputs(), c.reference()
    for name, x, y in zip(("O", "LSE", "dQ", "dK", "dV"), got, want):
        if name == "LSE":
            continue
        assert torch.isfinite(x).all(), name
        assert rel_err_fro(x.numpy(), y.numpy()) <= FRO[dtype], name


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_later_value_that_is_not_finite(lx, dtype):
    """Causal: a NaN in V at token 40 reaches the queries from 40 on, and no other; its gradient is hidden from nobody."""
    c = Call(lx, 1, 1, 1, 100, 100, 64, dtype, seed=10)
    c.V[0, 0, 40, 3] = math.nan
    c.forward()
    O = c.O[0, 0].double().cpu()
    assert torch.isfinite(O[:40]).all() and torch.isnan(O[40:, 3]).all()
    c = Call(lx, 1, 1, 1, 100, 100, 64, dtype, seed=10)
    c.dO[0, 0, 40, 3] = math.nan
    c.forward().backward()
    dQ, dK, dV = (t[0, 0].double().cpu() for t in (c.dQ, c.dK, c.dV))
    assert torch.isfinite(torch.cat([dQ[:40], dQ[41:]])).all() and torch.isnan(dQ[40]).all()
    assert torch.isfinite(dK[41:]).all() and torch.isfinite(dV[41:]).all()
    assert torch.isnan(dV[:41, 3]).all() and torch.isnan(dK[:41]).any(1).all()


def test_broadcast_keys(lx):
    """K and V of one batch entry for all (stride 0): every batch entry writes its own gradient."""
    c = Call(lx, 3, 4, 2, 130, 130, 64, "bf16", seed=11)
    c.K, c.V = c.K[:1].expand(3, -1, -1, -1), c.V[:1].expand(3, -1, -1, -1)
    c.check()


def test_packed_qkv(lx):
    c = Call(lx, 2, 4, 4, 140, 140, 64, "f16", seed=12)
    packed = torch.randn((2, 140, 3, 4, 64), generator=torch.Generator().manual_seed(4)).half().cuda()
    c.Q, c.K, c.V = (packed[:, :, i].transpose(1, 2) for i in range(3))
    c.check()


def test_offsets_beyond_32_bits(lx):
    """Batch entries 2^32 bytes and more apart, tokens 2^22 elements apart."""
    c = Call(lx, 2, 2, 2, 70, 70, 64, "bf16", seed=13)
    room = torch.empty((1 << 31) + (1 << 30), dtype=torch.bfloat16, device="cuda")
    for i, name in enumerate(("K", "V")):
        t = getattr(c, name)
        far = room[64 * i:].as_strided((2, 2, 70, 64), ((1 << 31) + 64, 128 + (1 << 21), 1 << 22, 1))
        far.copy_(t)
        setattr(c, name, far)
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_bits_and_other_streams(lx, dtype):
    a = Call(lx, 2, 4, 2, 333, 333, 64, dtype, seed=14, cap=5.0, slopes=True)
    b = Call(lx, 2, 4, 2, 333, 333, 64, dtype, seed=14, cap=5.0, slopes=True)
    a.forward().backward()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b.forward().backward()
    side.synchronize()
    for x, y in zip(a.outputs(), b.outputs()):
        assert torch.equal(x, y)


def test_graph(lx):
    c = Call(lx, 1, 4, 2, 200, 200, 128, "bf16", seed=15, cap=5.0)
    ws = [torch.empty(max(f(lx.LX_BF16, 1, 4, 2, 200, 200, 128), 256), dtype=torch.uint8, device="cuda")
          for f in (lx.lx_score_attn_fwd_workspace_bytes, lx.lx_score_attn_bwd_workspace_bytes)]

    def step():
        lx.lx_score_attn_fwd(c.Q, c.K, c.V, c.scale, True, c.O, c.LSE, workspace=ws[0], **c.rules)
        lx.lx_score_attn_bwd(c.Q, c.K, c.V, c.O, c.LSE, c.dO, c.scale, True, c.dQ, c.dK, c.dV, workspace=ws[1], **c.rules)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        c.Q.mul_(1.1)
        step()
        torch.cuda.synchronize()
        want = c.outputs()
        for t in (c.O, c.LSE, c.dQ, c.dK, c.dV):
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(c.outputs(), want):
            assert torch.equal(x, y), k


@pytest.mark.parametrize("cap,slopes", [(0.0, False), (3.0, True)])
def test_gradients_against_differences(lx, cap, slopes):
    """fp32: central differences of sum(O dO) along random directions.  The loss in steps of e = 1e-2 has an error of about
    e^2 (third derivatives of order one) + 2^-24 sqrt(S D) / e relative to a slope of order sqrt(S D): below 1e-3."""
    c = Call(lx, 1, 2, 1, 60, 60, 64, "f32", seed=16, cap=cap, slopes=slopes)
    c.forward().backward()
    for name, grad in (("Q", c.dQ), ("K", c.dK), ("V", c.dV)):
        x = getattr(c, name)
        v = torch.randn(x.shape, generator=torch.Generator().manual_seed(5)).cuda()
        v = v / v.norm() * 8
        loss = []
        for sign in (1, -1):
            setattr(c, name, x + sign * 1e-2 * v)
            c.forward()
            loss.append(float((c.O.double() * c.dO.double()).sum()))
        setattr(c, name, x)
        slope, want = (loss[0] - loss[1]) / 2e-2, float((grad.double() * v.double()).sum())
        assert abs(slope - want) <= 1e-3 * float(grad.double().norm() * v.double().norm()), (name, slope, want)


def test_refusals(lx):
    c = Call(lx, 2, 4, 2, 20, 20, 64, "bf16")

    def refused(status, **change):
        a = dict(Q=c.Q, K=c.K, V=c.V, scale=0.1, causal=True, O=c.O, LSE=c.LSE, cap=0.0)
        a.update(change)
        if status is None:
            with pytest.raises(AssertionError):
                lx.lx_score_attn_fwd(**a)
            return
        with pytest.raises(lx.LxError) as e:
            lx.lx_score_attn_fwd(**a)
        assert e.value.status == status
    refused(lx.LX_ERR_INVALID_ARG, cap=-1.0)
    refused(lx.LX_ERR_INVALID_ARG, cap=math.nan)
    refused(lx.LX_ERR_INVALID_ARG, scale=math.inf)
    refused(lx.LX_ERR_INVALID_ARG, key_lo=torch.zeros((2, 20), dtype=torch.int32, device="cuda"))
    refused(lx.LX_ERR_INVALID_ARG, K=c.K[:, :1].expand(-1, 3, -1, -1), V=c.V[:, :1].expand(-1, 3, -1, -1))   # 4 query heads, 3 key heads
    refused(lx.LX_ERR_INVALID_ARG, O=c.O[:1].expand(2, -1, -1, -1))
    refused(None, K=c.K[:, :, :19])
    refused(None, V=c.V.half())
    refused(None, O=c.O.float())
    refused(None, slopes=torch.zeros(3, device="cuda"))
    refused(None, q_start=torch.zeros(2, device="cuda"))
    refused(None, LSE=torch.zeros((2, 4, 21), device="cuda"))
    wide = torch.zeros((2, 4, 20, 96), dtype=torch.bfloat16, device="cuda")
    refused(lx.LX_ERR_UNSUPPORTED, Q=wide, K=wide[:, :2], V=wide[:, :2], O=wide.clone())
    with pytest.raises(lx.LxError) as e:
        lx.lx_score_attn_bwd(c.Q, c.K, c.V, c.O, c.LSE, c.dO, 0.1, True, c.dQ, c.dK, c.dV,
                             workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == lx.LX_ERR_WORKSPACE


@pytest.mark.parametrize("scale", [0.0, -0.2])
@pytest.mark.parametrize("D,cap", [(64, 0.0), (128, 5.0)])
def test_scales_that_are_not_positive(lx, scale, D, cap):
    c = Call(lx, 1, 2, 1, 90, 90, D, "bf16", seed=17, cap=cap)
    c.scale = scale
    c.check()
