"""Dropout and the norm of a sum with its residual (lx_dropout, lx_rms_norm_fwd, lx_rms_norm_bwd) against their definitions in 64 bits.

Tolerances.  One rounding to the element type is half a step, eps / 2 of the value (half precision: half of 2^-24 at least); a
rounding in 32 bits is U = 2^-24 of the value that it is made on.  A sum of n squares, at most 32 in a lane, 6 steps over
lanes and 4 or 16 wavefronts, is (32 + 6 + 16) U off, its root half of that, and quotient, root and products add 6: 40 U on y beside what h is off,
which is 3 U of |x c| + |r| (the factor, the product, the sum)."""
import math

import pytest
import torch

import block_reference as ref
from util import torch_dtype

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def half_step(dtype, value):
    """Half a step of the type at the value, with the type's smallest steps."""
    return torch.finfo(dtype).eps / 2 * value.abs() + torch.finfo(dtype).tiny * torch.finfo(dtype).eps / 2


def rows(g, T, d, dtype, gap=0, at=0, std=1.0):
    """[T, d] on the GPU, rows gap elements apart beyond d, from element `at` of a buffer that is NaN elsewhere."""
    buffer = torch.full((T * (d + gap) + at,), math.nan, dtype=torch_dtype(dtype))
    t = buffer[at:].view(T, d + gap)[:, :d]
    t.copy_((torch.randn((T, d), generator=g) * std).to(torch_dtype(dtype)))
    return buffer.cuda()[at:].view(T, d + gap)[:, :d]


def near(got, want, tolerance):
    off = (got.double().cpu() - want).abs()
    assert bool((off <= tolerance).all()), (float((off - tolerance).max()), float(off.max()))


SHAPES = [(1, 1), (3, 7), (5, 64), (2, 100), (9, 512), (4, 520), (7, 1024), (6, 2048), (3, 2056), (5, 4096), (2, 8191), (2, 16384), (1, 32768)]


@pytest.mark.parametrize("T,d", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_dropout(lx, T, d, dtype):
    g = torch.Generator().manual_seed(T + d)
    for gap, at, p, site in ((0, 0, 0.1, 0), (8, 0, 0.5, 7), (3, 1, 0.1, -1)):
        rng = torch.tensor([0x123456789ABCDEF, 41], dtype=torch.int64)
        x, r = rows(g, T, d, dtype, gap, at), rows(g, T, d, dtype, 2 * gap, at)
        f = ref.factors(T, d, p, int(rng[0]), int(rng[1]), site)
        xc, rc = x.double().cpu(), r.double().cpu()
        for residual in (None, r):
            out = rows(g, T, d, dtype, gap, 2 * at)
            lx.lx_dropout(x, out, p, rng.cuda(), site, residual=residual)
            want = xc * f + (0 if residual is None else rc)
            near(out, want, half_step(out.dtype, want) * (1 + 4 * U) + 4 * U * ((xc * f).abs() + rc.abs()))
            assert torch.equal(out.cpu() == 0, (f == 0) | (xc == 0)) if residual is None else True


def test_dropout_backward_is_the_same_call_and_nothing_is_dropped_at_zero(lx):
    g = torch.Generator().manual_seed(2)
    x, rng = rows(g, 33, 96, "f32"), torch.tensor([-5, 2 ** 40 + 3], dtype=torch.int64).cuda()
    one, out, back = torch.ones_like(x), torch.empty_like(x), torch.empty_like(x)
    lx.lx_dropout(x, out, 0.3, rng, 4)
    lx.lx_dropout(one, back, 0.3, rng, 4)
    near(out, x.double().cpu() * back.double().cpu(), 2 * U * x.double().cpu().abs() * 2)
    lx.lx_dropout(x, out, 0.0, None)
    assert torch.equal(out, x)
    x[0, 0], x[1, 1] = math.nan, math.inf        # in dropped places of a mask they have no effect
    lx.lx_dropout(one, back, 0.3, rng, 4)
    lx.lx_dropout(x, out, 0.3, rng, 4)
    assert torch.equal(torch.isfinite(out), torch.isfinite(x) | (back == 0))
    y = x.clone()
    lx.lx_dropout(y, y, 0.3, rng, 4)             # in place
    assert torch.equal(torch.nan_to_num(y, 9.0), torch.nan_to_num(out, 9.0))


def forward_case(lx, T, d, dtype, gap, at, p, with_residual, with_weight, seed=0):
    g = torch.Generator().manual_seed(seed + T * 7 + d)
    rng = torch.tensor([99 + seed, 7], dtype=torch.int64)
    x = rows(g, T, d, dtype, gap, at)
    r = rows(g, T, d, dtype, gap, at, 3.0) if with_residual else None
    w = (torch.randn(d, generator=g) * 0.3 + 1).to(torch_dtype(dtype)).cuda() if with_weight else None
    f = ref.factors(T, d, p, int(rng[0]), int(rng[1]), 3)
    h, y = ref.norm(x.cpu(), None if r is None else r.cpu(), None if w is None else w.cpu(), EPS, f)
    weight = torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
    off = 3 * U * ((x.double().cpu() * f).abs() + (0 if r is None else r.double().cpu().abs()))
    scale = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)
    return x, r, w, rng.cuda(), h, y, off, (40 * U * y.abs() + off * scale * weight.abs()) * (1 + 1e-5)


@pytest.mark.parametrize("T,d", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_norm(lx, T, d, dtype):
    for gap, at, p, res, wt in ((0, 0, 0.0, True, True), (8, 0, 0.1, True, True), (3, 1, 0.1, False, True), (0, 0, 0.0, False, False)):
        x, r, w, rng, h, y, off_h, off_y = forward_case(lx, T, d, dtype, gap, at, p, res, wt)
        H, Y = torch.full_like(x, math.nan), torch.full_like(x, math.nan)
        lx.lx_rms_norm_fwd(x, w, EPS, Y, residual=r, H=H, p=p, rng=rng if p else None, site=3)
        near(H, h, half_step(H.dtype, h) * (1 + 4 * U) + off_h)
        near(Y, y, half_step(Y.dtype, y) * (1 + 64 * U) + off_y)
        # in place: H in the residual's place, Y in x's
        x2, r2 = x.clone(), None if r is None else r.clone()
        lx.lx_rms_norm_fwd(x2, w, EPS, x2, residual=r2, H=r2, p=p, rng=rng, site=3)
        assert torch.equal(x2, Y) and (r is None or torch.equal(r2, H))


@pytest.mark.parametrize("T,d,group", [(1, 32, 32), (3, 7, 7), (5, 64, 32), (4, 520, 520), (7, 1024, 128), (16, 2048, 2048), (3, 2048, 512), (5, 4096, 256),
                                       (2, 4608, 64), (2, 16384, 128), (1, 32768, 32768)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_norm_in_8_bits(lx, T, d, group, dtype):
    for at, with_y in ((0, False), (1, True)):
        x, r, w, rng, h, y, _, off_y = forward_case(lx, T, d, dtype, 0, at, 0.1, True, True, seed=5)
        Y = torch.full_like(x, math.nan) if with_y else None
        buffer = torch.zeros(T * d + at, dtype=torch.uint8, device="cuda")
        Y8, scales = buffer[at:].view(torch.float8_e4m3fn).view(T, d), torch.full((T, d // group), math.nan, device="cuda")
        lx.lx_rms_norm_fwd(x, w, EPS, Y, residual=r, p=0.1, rng=rng, site=3, Y8=Y8, scales=scales)
        if with_y:
            near(Y, y, half_step(Y.dtype, y) * (1 + 64 * U) + off_y)
        groups, off = y.view(T, -1, group), off_y.view(T, -1, group)
        s = groups.abs().amax(-1) / 448
        near(scales, s, 2 * U * s + off.amax(-1) / 448)
        # a quotient is off by its own and the scale's error, its rounding by half a step: 2^-4 of the value, 2^-10 at least
        s = s[..., None]
        q = groups / s
        off = off / s + (off.amax(-1, keepdim=True) / 448 / s + 6 * U) * q.abs()
        near(Y8.float().view(T, -1, group), q, 2.0 ** -4 * (q.abs() + off) + 2.0 ** -10 + off)


def test_norm_of_rows_of_zeros_and_not_finite_values(lx):
    x = torch.zeros((4, 256), device="cuda")
    x[1, 5], x[2, 7], x[3] = math.nan, math.inf, 1.0
    Y, Y8, scales = torch.empty_like(x), torch.empty((4, 256), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((4, 2), device="cuda")
    lx.lx_rms_norm_fwd(x, None, EPS, Y, Y8=Y8, scales=scales)
    assert (Y[0] == 0).all() and (Y8[0].float() == 0).all() and (scales[0] == 2.0 ** -126).all()
    assert torch.isnan(Y[1]).all() and torch.isnan(scales[1]).all() and torch.isnan(Y8[1].float()).all()
    assert torch.isnan(Y[2, 7]) and (Y[2, :7] == 0).all() and torch.isnan(scales[2, 0]) and scales[2, 1] == 2.0 ** -126
    assert torch.isfinite(Y[3]).all() and (Y8[3].float() == 448).all()


@pytest.mark.parametrize("T,d", SHAPES + [(37, 768), (1500, 96), (5000, 40), (1030, 2056)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_norm_backward(lx, T, d, dtype):
    g = torch.Generator().manual_seed(T + d)
    few = T * d < 100000
    for gap, at, p, res, wt in ((0, 0, 0.1 if few else 0.0, True, True), (3, 1, 0.0, False, True), (8, 0, 0.0, True, False)):
        rng = torch.tensor([3, 4], dtype=torch.int64)
        h, dy = rows(g, T, d, dtype, gap, at, 2.0), rows(g, T, d, dtype, gap, at)
        dh = rows(g, T, d, dtype, gap, at) if res else None
        w = (torch.randn(d, generator=g) * 0.3 + 1).to(torch_dtype(dtype)).cuda() if wt else None
        f = ref.factors(T, d, p, 3, 4, 0)
        hc, dyc, wc = h.double().cpu(), dy.double().cpu(), torch.ones(d, dtype=torch.float64) if w is None else w.double().cpu()
        dX, dR, dW = ref.norm_back(dy.cpu(), h.cpu(), None if w is None else w.cpu(), EPS, None if dh is None else dh.cpu(), f)
        s = 1 / torch.sqrt((hc * hc).mean(-1, keepdim=True) + EPS)
        n = (hc * s).abs()
        # (54 + 6 roundings of sums of which the mean's are of its terms' sizes, the others of the parts of dR)
        off = 64 * U * (s * ((wc * dyc).abs() + n * ((wc * dyc).abs() * n).mean(-1, keepdim=True)) + (0 if dh is None else dh.double().cpu().abs()))
        gX, gR, gW = torch.full_like(h, math.nan), torch.full_like(h, math.nan), torch.full((d,), math.nan, device="cuda")
        lx.lx_rms_norm_bwd(dy, h, w, EPS, gX, dH=dh, dR=gR, dW=gW, p=p, rng=rng.cuda())
        near(gR, dR, half_step(gR.dtype, dR) * (1 + 4 * U) + off)
        near(gX, dX, half_step(gX.dtype, dX) * (1 + 4 * U) + (off + 2 * U * dR.abs()) * f)
        # rows of a workgroup, its wavefronts, a sixteenth of 1024 partial sums, sixteen of those; each term 45
        near(gW, dW, (T / 1024 + 4 + 64 + 16 + 45) * U * (dyc.abs() * n).sum(0))
        again = torch.empty_like(gW)
        gX2 = dy.clone()
        lx.lx_rms_norm_bwd(gX2, h, w, EPS, gX2, dH=dh, dW=again, p=p, rng=rng.cuda())       # in place, alone, the same bits
        assert torch.equal(again, gW) and torch.equal(gX2, gX)
        lx.lx_rms_norm_bwd(dy, h, w, EPS, None, dW=again)
        assert torch.equal(again, gW)


def test_many_rows(lx):
    """More rows than workgroups, each row like a call of its own."""
    g = torch.Generator().manual_seed(3)
    for T, d in ((20000, 64), (9000, 2304)):
        x, w = rows(g, T, d, "bf16"), torch.ones(d, dtype=torch.bfloat16, device="cuda")
        Y, dX, one = torch.empty_like(x), torch.empty_like(x), torch.empty((1, d), dtype=x.dtype, device="cuda")
        lx.lx_rms_norm_fwd(x, w, EPS, Y)
        lx.lx_rms_norm_bwd(Y, x, w, EPS, dX)
        for t in (0, 1, 4095, 4096, T // 2, T - 1):
            lx.lx_rms_norm_fwd(x[t:t + 1], w, EPS, one)
            assert torch.equal(one[0], Y[t])
            lx.lx_rms_norm_bwd(Y[t:t + 1], x[t:t + 1], w, EPS, one)
            assert torch.equal(one[0], dX[t])


def test_graph_and_streams(lx):
    """A captured step whose seed and step lie on the device, replayed with others, and on a stream of its own."""
    g = torch.Generator().manual_seed(4)
    x, r, w = rows(g, 50, 384, "f16"), rows(g, 50, 384, "f16"), torch.ones(384, dtype=torch.float16, device="cuda")
    rng = torch.tensor([1, 0], dtype=torch.int64, device="cuda")
    outs = [torch.empty_like(x) for _ in range(4)] + [torch.empty(384, device="cuda")]

    def step():
        lx.lx_rms_norm_fwd(x, w, EPS, outs[0], residual=r, H=outs[1], p=0.2, rng=rng, site=1)
        lx.lx_rms_norm_bwd(outs[0], outs[1], w, EPS, outs[2], dR=outs[3], dW=outs[4], p=0.2, rng=rng, site=1)
        rng[1:] += 1
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for i in range(4):
        at = rng.clone()
        x.mul_(1.1)
        if i % 2:
            step()
        else:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                step()
            torch.cuda.current_stream().wait_stream(side)
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        rng.copy_(at)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)) and int(rng[1]) == int(at[1]) + 1


def test_refusals(lx):
    x, rng = torch.zeros((4, 64), device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    for bad in (dict(out=x.cpu()), dict(rng=rng.cpu()), dict(X=x.cpu()), dict(residual=x.cpu())):
        a = {**dict(X=x, out=x, rng=rng, residual=None), **bad}
        with pytest.raises(AssertionError):
            lx.lx_dropout(a["X"], a["out"], 0.1, a["rng"], residual=a["residual"])
    with pytest.raises(lx.LxError):
        lx.lx_dropout(x, x, 1.0, rng)
    with pytest.raises(lx.LxError):
        lx.lx_rms_norm_fwd(x, None, EPS, None)
    with pytest.raises(lx.LxError) as e:
        lx.lx_rms_norm_bwd(x, x, None, EPS, x, dW=torch.empty(64, device="cuda"), workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == lx.LX_ERR_WORKSPACE


def test_dropout_of_the_longest_rows(lx):
    """d = 2^31 - 1: whose runs are more than an int's sum with 7 can count; elements past 2^32."""
    T, d = 3, 2 ** 31 - 1
    x, rng = torch.ones((T, d), dtype=torch.bfloat16, device="cuda"), torch.tensor([77, 5], dtype=torch.int64, device="cuda")
    out = torch.full_like(x, math.nan)
    lx.lx_dropout(x, out, 0.5, rng, 9)
    runs = 2 ** 28
    for t in range(T):
        for j in (0, 1, 12345678, runs - 2, runs - 1):
            n = t * runs + j
            words = ref.philox((n & ref.MASK, n >> 32, 9, 5), (77, 0))
            want = [0.0 if words[i // 2] >> 16 * (i % 2) & 0xFFFF < 32768 else 2.0 for i in range(min(8, d - 8 * j))]
            assert out[t, 8 * j:8 * j + 8].tolist() == want, (t, j)
        kept = sum(float((part == 2).sum()) for part in out[t].split(2 ** 28)) / d
        assert abs(kept - 0.5) < 6 * 0.5 / math.sqrt(d)
        assert all(bool(((part == 0) | (part == 2)).all()) for part in out[t].split(2 ** 28))


FILL = 7.0


class Strided:
    """[T, d] with rows `gap` elements apart beyond d, from element `at` of a buffer that is FILL elsewhere; holds `t`, or FILL."""

    def __init__(self, T, d, dtype, gap, at, t=None):
        self.buffer = torch.full((T * (d + gap) + at + 16,), FILL, dtype=dtype, device="cuda")
        self.rows = self.buffer[at:at + T * (d + gap)].view(T, d + gap)[:, :d]
        if t is not None:
            self.rows.copy_(t)

    def equal(self, want):
        """The rows are `want`, and the buffer is as it was elsewhere."""
        got = self.rows.clone()
        self.rows.fill_(FILL)
        return torch.equal(got, want) and bool((self.buffer == FILL).all())


# of x, residual, H, Y (and in the backward pass dY, H, dH, dX, dR): all apart from each other, in accesses of 16 bytes and otherwise
LAYOUTS = {"aligned": ((8, 0), (16, 8), (24, 16), (40, 0), (64, 8)), "odd": ((3, 1), (5, 2), (7, 3), (1, 5), (9, 4)), "rows": ((1, 0), (8, 1), (0, 3), (2, 0), (0, 0))}


@pytest.mark.parametrize("T,d", [(1, 8), (3, 7), (5, 64), (4, 520), (3, 2056), (2, 4096), (2, 8191), (2, 16392)], ids=str)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_layouts_of_their_own(lx, T, d, layout, dtype):
    """Every tensor in a layout of its own, outputs too, and in place: the bits of contiguous calls, which are near the definition, and nothing between the rows."""
    places, dt, p = LAYOUTS[layout], torch_dtype(dtype), 0.1
    x, r, w, rng, h, y, off_h, off_y = forward_case(lx, T, d, dtype, 0, 0, p, True, True, seed=9)
    H, Y = torch.full_like(x, math.nan), torch.full_like(x, math.nan)
    lx.lx_rms_norm_fwd(x, w, EPS, Y, residual=r, H=H, p=p, rng=rng, site=3)
    near(H, h, half_step(dt, h) * (1 + 4 * U) + off_h)
    near(Y, y, half_step(dt, y) * (1 + 64 * U) + off_y)

    def at(k, t=None):
        return Strided(T, d, dt, *places[k], t)
    sx, sr, sh, sy = at(0, x), at(1, r), at(2), at(3)
    lx.lx_rms_norm_fwd(sx.rows, w, EPS, sy.rows, residual=sr.rows, H=sh.rows, p=p, rng=rng, site=3)
    assert sh.equal(H) and sy.equal(Y) and sx.equal(x) and sr.equal(r)
    sx, sr = at(0, x), at(1, r)
    lx.lx_rms_norm_fwd(sx.rows, w, EPS, sx.rows, residual=sr.rows, H=sr.rows, p=p, rng=rng, site=3)      # in place
    assert sx.equal(Y) and sr.equal(H)
    sx, sr = at(0, x), at(1, r)
    lx.lx_rms_norm_fwd(sx.rows, w, EPS, sr.rows, residual=sr.rows, H=sx.rows, p=p, rng=rng, site=3)      # ... the other way round
    assert sx.equal(H) and sr.equal(Y)
    # one row for all, as the residual and as dY
    lx.lx_rms_norm_fwd(x, w, EPS, Y, residual=r[:1].expand(T, d).contiguous(), H=H, p=p, rng=rng, site=3)
    sy, sh = at(3), at(2)
    lx.lx_rms_norm_fwd(x, w, EPS, sy.rows, residual=r[:1].expand(T, d), H=sh.rows, p=p, rng=rng, site=3)
    assert sh.equal(H) and sy.equal(Y)

    dropped, out = torch.full_like(x, math.nan), at(3)
    lx.lx_dropout(x, dropped, p, rng, 3, residual=r)
    sx, sr = at(0, x), at(1, r)
    lx.lx_dropout(sx.rows, out.rows, p, rng, 3, residual=sr.rows)
    lx.lx_dropout(sx.rows, sr.rows, p, rng, 3, residual=sr.rows)
    assert out.equal(dropped) and sr.equal(dropped) and sx.equal(x)

    for dY in (y.to(dt).cuda(), y[:1].to(dt).cuda().expand(T, d)):
        dX, dR, dW, dW2 = torch.full_like(x, math.nan), torch.full_like(x, math.nan), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        lx.lx_rms_norm_bwd(dY.contiguous(), H, w, EPS, dX, dH=r, dR=dR, dW=dW, p=p, rng=rng, site=3)
        sdy, sh, sdh, sdx, sdr = at(0, dY), at(1, H), at(2, r), at(3), at(4)
        lx.lx_rms_norm_bwd(sdy.rows if dY.stride(0) else dY, sh.rows, w, EPS, sdx.rows, dH=sdh.rows, dR=sdr.rows, dW=dW2, p=p, rng=rng, site=3)
        assert sdx.equal(dX) and sdr.equal(dR) and torch.equal(dW, dW2) and sh.equal(H) and sdh.equal(r)
        sdy, sh, sdh = at(0, dY), at(1, H), at(2, r)
        lx.lx_rms_norm_bwd(sdy.rows, sh.rows, w, EPS, sdy.rows, dH=sdh.rows, dR=sdh.rows, dW=dW2, p=p, rng=rng, site=3)      # in place of dY and dH
        assert sdy.equal(dX) and sdh.equal(dR) and torch.equal(dW, dW2)
        sdy, sh = at(0, dY), at(1, H)
        lx.lx_rms_norm_bwd(sdy.rows, sh.rows, w, EPS, sh.rows, dH=r, dR=sdy.rows, dW=dW2, p=p, rng=rng, site=3)               # ... of H and dY
        assert sh.equal(dX) and sdy.equal(dR) and torch.equal(dW, dW2)
