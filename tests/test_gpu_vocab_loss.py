"""The loss over a vocabulary and its gradients (lx_vocab_loss) against the definition in 64 bits.

Tolerances.  U = 2^-24.  z is a sum of d exact products, 32 to an instruction: off by Z = (d / 32 + 32) 2 U sum |x w| at most.  A loss is off by what
z moves it, 2 Z (1 - p), p the target's probability, by the sums and exponentials, 300 U of the same, and by its own roundings, 8 U of it.
An element of G is off by its factor, 2 Z + 300 U, its rounding in half precision, 2^-11, and the one to the element type, eps / 2; or, where that
is half precision, by half of the smallest step, 2^-25, of the scaled values, the largest weight standing at 2^14 (2^13 after the power of
two): 2^-38 of that weight; exponentials and products below 2^-126 vanish.  In the target's column the rounding to the element type is made up: in dX in
fp32, in dW by another element of the type, of at most eps / 2 of it, which is rounded in turn.  dX and dW add products of those, off by (n / 32 + 32) 2 U of their sizes, and are rounded."""
import math

import pytest
import torch

import block_reference as ref
from util import FRO, torch_dtype

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def make(T, d, V, dtype, ignored=0.2, weighted=False, lift=8.0, seed=0, gap=0, at=0):
    """X (rows gap apart, from element `at` of a buffer), W, targets, weights; what ignored tokens hold is NaN."""
    g = torch.Generator().manual_seed(seed + T + d + V)
    dt = torch_dtype(dtype)
    W = (torch.randn((V, d), generator=g) * 2 * d ** -0.5).to(dt)
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    X = torch.randn((T, d), generator=g) + lift * torch.rand((T, 1), generator=g) * 0.25 * W[targets.long()].float()
    out = torch.rand(T, generator=g) < ignored
    X[out] = math.nan
    targets[out] = torch.tensor([-100, -1, V, 2 ** 31 - 1], dtype=torch.int32)[torch.randint(0, 4, (T,), generator=g)][out]
    weights = torch.rand(T, generator=g) * 3 - 0.5 if weighted else None
    buffer = torch.full((T * (d + gap) + at,), math.nan, dtype=dt)
    buffer[at:].view(T, d + gap)[:, :d] = X.to(dt)
    return buffer.cuda()[at:].view(T, d + gap)[:, :d], W.cuda(), targets.cuda(), None if weights is None else weights.cuda()


def check(X, W, targets, weights, loss, lse, dX, dW):
    """Against the definition, by the tolerances above."""
    x, w, t = X.cpu().double(), W.cpu().double(), targets.cpu()
    T, V, d = x.shape[0], w.shape[0], w.shape[1]
    held = (t >= 0) & (t < V)
    x = torch.where(held[:, None], x, 0.0)
    wt = torch.ones(T, dtype=torch.float64) if weights is None else weights.cpu().double()
    rloss, rlse, rdX, rdW = ref.vocab_loss(X.cpu(), W.cpu(), t, None if weights is None else weights.cpu())
    Z = (d / 32 + 32) * 2 * U * (x.abs() @ w.abs().t()).amax(-1)
    P = torch.exp(x @ w.t() - rlse[:, None]) * held[:, None]
    tt = t.long().clamp(0, V - 1)
    p = P.gather(1, tt[:, None])[:, 0]
    rest = torch.where(held, -torch.expm1(-rloss), 0.0)
    assert bool(((loss.cpu().double() - rloss).abs() <= (2 * Z + 300 * U) * rest + 8 * U * rloss + V * 2.0 ** -126).all())
    if lse is not None:
        assert bool(((lse.cpu().double() - rlse).abs() <= held * (Z + 300 * U + 4 * U * rlse.abs())).all())
    eps = torch.finfo(X.dtype).eps / 2 if X.dtype != torch.float32 else 0.0      # (2 U of its own below)
    tiny = torch.finfo(X.dtype).tiny * torch.finfo(X.dtype).eps / 2       # half of the smallest step of what is written
    G = (P.scatter(1, tt[:, None], 0.0) + torch.zeros_like(P).scatter(1, tt[:, None], (rest * held)[:, None])) * wt.abs()[:, None]
    rounding = torch.full_like(G, eps + (2.0 ** -11 if eps else 0.0)).scatter_(1, tt[:, None], eps * eps * 1.01)
    off = G * (rounding + 2 * Z[:, None] + 300 * U) + (held * wt.abs())[:, None] * 2.0 ** -125
    if X.dtype == torch.float16:
        off = off + held[:, None] * 2.0 ** -38 * float((wt.abs() * held).max())
    for got, want, other, n in ((dX, rdX, w, V), (dW, rdW, x, T)):
        if got is None:
            continue
        a, g = (G, off) if got is dX else (G.t(), off.t())
        last = 2 * U if got.dtype == torch.float32 else eps
        limit = g @ other.abs() + (n / 32 + 32) * 2 * U * (a @ other.abs()) + last * want.abs() * 1.01 + tiny
        far = (got.cpu().double() - want).abs()
        assert bool((far <= limit).all()), (float((far / limit.clamp(min=1e-30)).max()), float(far.max()))
        norm = float(want.norm())
        if norm > 0 and want.numel() > 1000:
            gate = FRO[{torch.bfloat16: "bf16", torch.float16: "f16", torch.float32: "f32"}[X.dtype]]
            assert float(far.norm()) <= gate * norm, float(far.norm()) / norm


def call(lx, X, W, targets, weights, dX=True, dW=None, workspace=None):
    T = X.shape[0]
    loss, lse = (torch.full((T,), math.nan, device="cuda") for _ in range(2))
    dX = torch.full_like(X, math.nan) if dX is True else dX
    dW = torch.full(W.shape, math.nan, dtype=dW, device="cuda") if isinstance(dW, torch.dtype) else dW
    lx.lx_vocab_loss(X, W, targets, loss, lse=lse, weights=weights, dX=dX, dW=dW, workspace=workspace)
    return loss, lse, dX, dW


SIZES = [(1, 64, 1), (1, 64, 2), (3, 64, 63), (5, 128, 64), (64, 64, 65), (65, 192, 127), (257, 256, 129), (300, 320, 1000), (40, 64, 20000),
         (130, 768, 9001), (700, 512, 3000), (16, 2048, 5003), (1030, 128, 515)]


@pytest.mark.parametrize("T,d,V", SIZES, ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_sizes(lx, T, d, V, dtype):
    args = make(T, d, V, dtype, ignored=0.2 if T > 1 else 0.0)
    loss, lse, dX, dW = call(lx, *args, dW=torch_dtype(dtype))
    check(*args, loss, lse, dX, dW)
    # the same bits without gradients and into fp32; with dX alone bfloat16 exponentials are kept otherwise
    one, two, _, _ = call(lx, *args, dX=None)
    assert torch.equal(one, loss) and torch.equal(two, lse)
    check(*args, *call(lx, *args))
    out = call(lx, *args, dX=None, dW=torch.float32)
    check(*args, out[0], None, None, out[3])
    assert torch.equal(out[3].to(dW.dtype), dW)
    assert dtype != "f32" or torch.equal(call(lx, *args)[2], dX)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("gap,at", [(8, 0), (5, 1), (0, 3)])
def test_strides_weights_and_certain_tokens(lx, dtype, gap, at):
    args = make(150, 256, 2000, dtype, weighted=True, lift=60.0, gap=gap, at=at)       # logits of the targets up to 60 above the others
    dX = torch.full((150 * (256 + 2 * gap) + at,), 7.0, dtype=args[0].dtype, device="cuda")[at:].view(150, -1)
    for out in (None, torch.float32):
        loss, lse, got, dW = call(lx, *args, dX=dX[:, :256], dW=out)
        check(*args, loss, lse, got, dW)
    assert bool((dX[:, 256:] == 7.0).all())            # between the rows nothing is written
    assert float(loss[loss > 0].min()) < 1e-10


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,tokens", [(700, 256), (513, 512), (1000, 300)])
def test_pieces(lx, dtype, T, tokens):
    """A smaller workspace: more pieces, the last of another length."""
    args = make(T, 192, 700, dtype, weighted=True)
    code = {"bf16": lx.LX_BF16, "f16": lx.LX_F16, "f32": lx.LX_F32}[dtype]
    for out in (torch.float32, torch_dtype(dtype)):
        size = lx.lx_vocab_loss_workspace_bytes(code, T, 192, 700, lx.LX_GRAD_X | lx.LX_GRAD_W, lx.LX_F32 if out == torch.float32 else code, tokens)
        guard = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        got = call(lx, *args, dW=out, workspace=guard[:size])
        check(*args, *got)
        assert bool((guard[size:] == 0xA5).all())
        again = call(lx, *args, dW=out, workspace=guard[:size])
        assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,d,V", [(1, 64, 3), (2, 128, 700), (17, 192, 1), (33, 256, 4100), (63, 64, 130), (64, 1024, 999)], ids=str)
def test_few_tokens_without_gradients(lx, dtype, T, d, V):
    """Up to 64 tokens are read where they lie, from wherever that is."""
    for gap, at, ignored in ((0, 0, 0.3), (64, 0, 0.0), (8, 8, 0.7), (3, 1, 0.3)):
        args = make(T, d, V, dtype, ignored=ignored, gap=gap, at=at)
        loss, lse, _, _ = call(lx, *args, dX=None)
        check(*args, loss, lse, None, None)
    lone = torch.full((T,), math.nan, device="cuda")
    lx.lx_vocab_loss(*args[:3], lone)                  # without lse
    assert torch.equal(lone, loss)


@pytest.mark.parametrize("dtype,grads", [("bf16", "x"), ("bf16", "xw"), ("f16", "xw"), ("bf16", "")])
def test_largest_vocabulary(lx, dtype, grads):
    """2^20 rows, by the narrowest tiles and by wide ones."""
    for T in (5, 70):
        args = make(T, 64, 1 << 20, dtype, ignored=0.0)
        out = call(lx, *args, dX=True if grads else None, dW=torch.float32 if "w" in grads and T == 5 else None)
        check(*args, *out)


@pytest.mark.parametrize("T,d,V", [(4097, 64, 33), (65537, 64, 70)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_tokens(lx, T, d, V, dtype):
    """More tokens than a gathering workgroup each would do for, more than a piece holds."""
    args = make(T, d, V, dtype, ignored=0.3)
    out = call(lx, *args, dX=True, dW=torch.float32)
    check(*args, *out)


@pytest.mark.parametrize("T,V,few", [(700, 20000, 1), (700, 20000, 3), (1500, 300, 2), (3000, 1000, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_few_different_targets(lx, T, V, few, dtype):
    """Many tokens with the same targets, whose tiles of the vocabulary have many more steps than the others; pieces of 256 tokens too."""
    X, W, targets, weights = make(T, 128, V, dtype, weighted=True)
    held = (targets >= 0) & (targets < V)
    targets[held] = targets[held] % few * (V // few)
    args = X, W, targets, weights
    check(*args, *call(lx, *args, dX=True, dW=torch.float32))
    check(*args, *call(lx, *args, dX=None, dW=X.dtype))
    kind = {"bf16": lx.LX_BF16, "f16": lx.LX_F16}[dtype]
    size = lx.lx_vocab_loss_workspace_bytes(kind, T, 128, V, lx.LX_GRAD_W, lx.LX_F32, 256)
    check(*args, *call(lx, *args, dX=None, dW=torch.float32, workspace=torch.empty(size, dtype=torch.uint8, device="cuda")))


@pytest.mark.parametrize("T,d,V", [(1, 1152, 9001), (17, 448, 40000), (63, 64, 3), (64, 576, 4097)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_few_tokens(lx, T, d, V, dtype):
    """Up to 64 tokens, in rows that lie at 16 bytes and elsewhere: every gradient, and rows without a target."""
    for gap, at in ((0, 0), (8, 8), (1, 0)):
        args = make(T, d, V, dtype, ignored=0.3 if T > 1 else 0.0, weighted=True, gap=gap, at=at)
        held = (args[2] >= 0) & (args[2] < V)
        for dX, dW in ((True, None), (None, args[0].dtype), (True, torch.float32)):
            out = call(lx, *args, dX=dX, dW=dW)
            check(*args, *out)
            assert not bool(out[0][~held].any()) and (dX is None or not bool(out[2][~held].any()))


def test_rows_past_4_gib(lx):
    """As many tokens of the widest rows as a piece holds: dW against products in 64 bits, a few rows at a time."""
    T, d, V = 65536, 32768, 3
    g = torch.Generator(device="cuda").manual_seed(5)
    W = (torch.randn((V, d), generator=g, device="cuda") * 2 * d ** -0.5).bfloat16()
    X = torch.randn((T, d), generator=g, device="cuda", dtype=torch.bfloat16)
    targets = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    loss, _, _, dW = call(lx, X, W, targets, None, dX=None, dW=torch.float32)
    want, w = torch.zeros((V, d), dtype=torch.float64, device="cuda"), W.double()
    for t in range(0, T, 4096):
        x = X[t:t + 4096].double()
        z = x @ w.t()
        lse = z.logsumexp(-1)
        G = torch.exp(z - lse[:, None])
        rows = torch.arange(x.shape[0], device="cuda")
        at = targets[t:t + 4096].long()
        assert float((loss[t:t + 4096] - (lse - z[rows, at])).abs().max()) < 1e-4
        G[rows, at] -= 1
        want += G.t() @ x
    assert float((dW - want).norm()) <= FRO["bf16"] * float(want.norm())


@pytest.mark.parametrize("grads", ["x", "xw", ""])
def test_widest_rows(lx, grads):
    args = make(70, 32768, 200, "bf16", ignored=0.1)
    out = call(lx, *args, dX=True if grads else None, dW=torch.float32 if "w" in grads else None)
    check(*args, *out)


def test_no_targets(lx):
    X, W, targets, _ = make(100, 64, 300, "bf16", ignored=1.0)
    loss, lse, dX, dW = call(lx, X, W, targets, None, dW=torch.bfloat16)
    assert all(bool((t == 0).all()) for t in (loss, lse, dX, dW))
    for T in (50, 100):
        loss, lse, _, _ = call(lx, X[:T], W, targets[:T], None, dX=None)
        assert bool((loss == 0).all()) and bool((lse == 0).all())


def test_few_targets_at_the_end(lx):
    X, W, targets, _ = make(3000, 128, 1500, "f16", ignored=0.0)
    targets[:2990] = -100
    X[:2990] = math.inf
    out = call(lx, X, W, targets, None, dW=torch.float16)
    check(X, W, targets, None, *out)


def test_values_that_are_not_finite(lx):
    X, W, targets, _ = make(70, 64, 500, "bf16", ignored=0.0)
    X[7, 3], X[9, 0] = math.nan, math.inf
    loss, lse, dX, _ = call(lx, X, W, targets, None)
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[7] = bad[9] = True
    assert torch.equal(~torch.isfinite(loss), bad) and torch.equal(~torch.isfinite(dX).all(1), bad)
    clean = X.clone()
    clean[7] = clean[9] = 0
    want = call(lx, clean, W, targets, None)
    assert torch.equal(loss[~bad], want[0][~bad]) and torch.equal(dX[~bad], want[2][~bad])


def test_large_logits(lx):
    """Logits in the thousands: exponentials only of differences."""
    X, W, targets, _ = make(60, 64, 400, "bf16", ignored=0.1)
    X = torch.where(torch.isnan(X), X, X * 500)
    check(X, W, targets, None, *call(lx, X, W, targets, None, dW=torch.float32))
    check(X, W, targets, None, *call(lx, X, W, targets, None))


@pytest.mark.parametrize("V", [200, 1000, 5000])
def test_targets_far_below_the_others(lx, V):
    """Logits 40 to 120 above the target's in one place, in many or in all: on both sides of the limit from which a unit's exponentials are no
    longer kept relative to the target."""
    X, W, targets, _ = make(90, 64, V, "bf16", ignored=0.1, lift=0.0)
    for places in (1, V // 3, V):
        above, w = X.clone(), W.clone()
        w[:, 0] = 0                              # one feature sets a token's places apart
        w[:places, 0] = 1
        targets[(targets >= 0) & (targets < V)] = V - 1
        if places == V:
            w[V - 1, 0] = 0
        above[:, 0] = torch.where(torch.isnan(X[:, 0]), X[:, 0], torch.linspace(40, 120, 90, device="cuda").to(X.dtype))
        check(above, w, targets, None, *call(lx, above, w, targets, None))


def test_weights_far_apart_in_half_precision(lx):
    X, W, targets, _ = make(90, 64, 400, "f16", ignored=0.0)
    weights = torch.logspace(-6, 3, 90).cuda()
    check(X, W, targets, weights, *call(lx, X, W, targets, weights, dW=torch.float32))


def test_gradients_against_differences(lx):
    """The gradients as written against differences of the definition's loss."""
    X, W, targets, weights = make(6, 64, 40, "bf16", ignored=0.3, weighted=True, lift=1.0)
    _, _, dX, dW = call(lx, X, W, targets, weights, dW=torch.float32)
    x, w, t, wt = torch.nan_to_num(X.cpu().double()), W.cpu().double(), targets.cpu(), weights.cpu()

    def total(x, w):
        return float((ref.vocab_loss(x, w, t, None)[0] * wt.double()).sum())
    g = torch.Generator().manual_seed(1)
    for _ in range(8):
        a, b = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64)
        h = 1e-5
        for along, slope, size in (((a, 0 * b), float((dX.cpu().double() * a).sum()), (dX.cpu().double() * a).norm()),
                                   ((0 * a, b), float((dW.cpu().double() * b).sum()), (dW.cpu().double() * b).norm())):
            want = (total(x + h * along[0], w + h * along[1]) - total(x - h * along[0], w - h * along[1])) / (2 * h)
            # elements are off by three roundings of 2^-8 at most, in either direction: six deviations of their sum
            assert abs(slope - want) <= 6 * 3 * 2.0 ** -8 * float(size) / math.sqrt(3)


@pytest.mark.parametrize("T", [300, 40])
def test_graph_and_streams(lx, T):
    args = list(make(T, 128, 1000, "bf16", weighted=True))
    outs = [torch.empty(T, device="cuda"), torch.empty_like(args[0]), torch.empty_like(args[1])]

    def step():
        lx.lx_vocab_loss(*args[:3], outs[0], weights=args[3], dX=outs[1], dW=outs[2])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    side = torch.cuda.Stream()
    for i in range(4):
        args[2].copy_(torch.roll(args[2], 1 + i))
        args[0].copy_(torch.nan_to_num(args[0]) * 1.01)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals(lx):
    X, W, targets, _ = make(4, 64, 100, "bf16", ignored=0.0)
    loss = torch.empty(4, device="cuda")
    for bad in (dict(W=W.cpu()), dict(W=W.half()), dict(W=W[:, :32]), dict(targets=targets.long()), dict(targets=targets[:3]), dict(loss=loss.double()),
                dict(dX=X[:3]), dict(dX=X.float()), dict(dW=W[:50]), dict(dW=W.half()), dict(weights=loss[:2]), dict(lse=loss.cpu())):
        a = {**dict(X=X, W=W, targets=targets, loss=loss), **bad}
        with pytest.raises(AssertionError):
            lx.lx_vocab_loss(**a)
    with pytest.raises(lx.LxError) as e:
        lx.lx_vocab_loss(X, W, targets, loss, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == lx.LX_ERR_WORKSPACE
    with pytest.raises(lx.LxError) as e:
        lx.lx_vocab_loss(X[:, :48], W[:, :48].contiguous(), targets, loss)
    assert e.value.status == lx.LX_ERR_UNSUPPORTED


@pytest.mark.parametrize("T", [9, 100])
@pytest.mark.parametrize("dX,dW", [(True, None), (True, torch.bfloat16), (None, torch.float32)])
def test_words_far_below_their_neighbours(lx, T, dX, dW):
    """bfloat16: words 20 to 82 below another one among 32, which alone feed their rows of dW and columns of dX.  Limits as above, but for what
    exponentials lose that stand 2^-79 and more below their unit's largest: 2^-9 instead of 2^-11."""
    d, V = 64, 160
    g = torch.Generator().manual_seed(T)
    fall = torch.full((V,), 5.0)
    fall[0], fall[V - 1], fall[1:32] = 0.0, 0.0, 22 + 2 * torch.arange(31.0) - 2
    W, X = torch.zeros((V, d)), torch.randn((T, d), generator=g)
    W[:, 0], X[:, 0] = -fall, 1.0
    W[torch.arange(1, 32), torch.arange(1, 32)], X[:, 1:32] = 1.0, 0.0          # z = -fall, exactly
    targets, weights = torch.full((T,), V - 1, dtype=torch.int32), torch.rand(T, generator=g) + 0.5
    args = X.bfloat16().cuda(), W.bfloat16().cuda(), targets.cuda(), weights.cuda()
    x, w, wt = args[0].double().cpu(), args[1].double().cpu(), weights.double()
    loss, lse, gX, gW = call(lx, *args, dX=dX, dW=dW)
    rloss, rlse, rdX, rdW = ref.vocab_loss(x, w, targets, weights)
    assert float((loss.double().cpu() - rloss).abs().max()) < 1e-5 and float((lse.double().cpu() - rlse).abs().max()) < 1e-5
    Z, eps = (d / 32 + 32) * 2 * U * float((x.abs() @ w.abs().t()).max()), 2.0 ** -8
    G = torch.exp(x @ w.t() - rlse[:, None]) * wt[:, None]
    G[:, V - 1] = (1 - torch.exp(-rloss)) * wt
    rounding = eps + torch.where(fall < 54.8, 2.0 ** -11, 2.0 ** -9).double()
    rounding[V - 1] = eps * eps * 1.01
    off = G * (rounding + 2 * Z + 300 * U) + wt[:, None] * 2.0 ** -125
    for got, want, a, e, other, n in ((gX, rdX, G, off, w, V), (gW, rdW, G.t(), off.t(), x, T)):
        if got is None:
            continue
        last = eps if got.dtype == torch.bfloat16 else 2 * U
        limit = e @ other.abs() + (n / 32 + 32) * 2 * U * (a @ other.abs()) + last * want.abs() * 1.01 + 2.0 ** -134
        far = (got.double().cpu() - want).abs()
        assert bool((far <= limit).all()), (float((far / limit.clamp(min=1e-44)).max()), float(far.max()))
        assert bool((got[:, 1:32] if got is gX else got[1:32, 32:]).ne(0).all())


def test_units_far_above_the_target_are_rounded_once(lx):
    """dX alone in bfloat16, words in units of their own 75 to 97 above the target's, below another unit's that stand higher still: each of them
    feeds a column of dX by itself, off by its own rounding and dX's and no third one."""
    T, d, V = 300, 64, 1024
    W, X = torch.zeros((V, d)), torch.zeros((T, d))
    X[:, 0] = 1 + torch.arange(T) % 32 / 128.0
    W[:V - 128, 0] = 60.0
    W[0, 0] = 80.0                               # the highest unit; the target's, 0, is in the last one
    words = 384 + torch.arange(1, 64)
    W[words, 0] = 75.0 + (torch.arange(1, 64) % 5) / 2
    W[words, torch.arange(1, 64)] = 1.0
    targets = torch.full((T,), V - 1, dtype=torch.int32)
    args = X.bfloat16().cuda(), W.bfloat16().cuda(), targets.cuda(), (0.5 + torch.arange(T) / T).cuda()
    out = call(lx, *args)
    check(*args, *out)
    dX, want = out[2].double().cpu()[:, 1:], ref.vocab_loss(args[0].cpu(), args[1].cpu(), targets, args[3].cpu())[2][:, 1:]
    # two roundings to bfloat16; z of one product, its difference to the reference and the powers of two 2^-24 of 100 each; sums and factors 300 U
    limit = (2 * 2.0 ** -8 + 2.0 ** -16 + 4 * 100 * U + 300 * U) * want.abs()
    assert bool(((dX - want).abs() <= limit).all()), float(((dX - want).abs() / want.abs()).max()) * 2 ** 8


def test_small_weights_of_tokens_far_below(lx):
    """Targets 60 below all others, weights whose product with the others' sum is far below the smallest normal number; and large rows of W."""
    X, W, targets, _ = make(90, 64, 5000, "bf16", ignored=0.1, lift=0.0)
    held = (targets >= 0) & (targets < 5000)
    targets[held] = 4999
    W[:, 0], W[4999, 0] = 1.0, 0.0
    X[:, 0] = torch.where(torch.isnan(X[:, 0]), X[:, 0], 60.0)
    weights = torch.full((90,), 2.0 ** -46, device="cuda")
    check(X, W, targets, weights, *call(lx, X, W, targets, weights))
    # a column that the logits do not see, 2^30 in every row of W: its gradient is 0, and the other columns' the same bits as with 0 there.  (A row of G adds up
    # to 0 exactly; what is computed adds up to two roundings of its elements at most, which are 2 in all, so that no share of its norm can be asked for.)
    X[:, 63], W[:, 63] = torch.where(torch.isnan(X[:, 0]), X[:, 0], 0.0), 2.0 ** 30
    large = call(lx, X, W, targets, weights)[2]
    W[:, 63] = 0.0
    none = call(lx, X, W, targets, weights)[2]
    assert torch.equal(large[:, :63], none[:, :63]) and float(large[:, 63].abs().max()) <= 2.0 ** -46 * 2.0 ** 30 * 2 * 2 * 2.0 ** -8


@pytest.mark.parametrize("T,d,V", [(1, 64, 130), (5, 192, 700), (64, 448, 4100), (65, 64, 300), (300, 320, 1000)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_layouts_of_dX(lx, T, d, V, dtype):
    """dX in a layout that is not X's, X's rows one for all: the gradients of contiguous calls, and nothing between the rows."""
    args = make(T, d, V, dtype, ignored=0.3 if T > 1 else 0.0, weighted=True)
    held = ((args[2] >= 0) & (args[2] < V))[:, None]
    for gap, at in ((8, 0), (24, 8), (3, 1), (0, 5)):
        buffer = torch.full((T * (d + gap) + at + 16,), 7.0, dtype=args[0].dtype, device="cuda")
        rows = buffer[at:at + T * (d + gap)].view(T, d + gap)[:, :d]
        for dW in (None, torch.float32):
            out = call(lx, *args, dX=rows, dW=dW)
            check(*args, *out)
            assert not bool(torch.where(held, 0.0, rows).any())
            rows.fill_(7.0)
            assert bool((buffer == 7.0).all())
            one = args[0][int(held[:, 0].nonzero()[0])].clone()[None].expand(T, d)
            out = call(lx, one, *args[1:], dX=rows, dW=dW)
            check(one, *args[1:], *out)
            rows.fill_(7.0)
            assert bool((buffer == 7.0).all())


def test_units_far_below_one_that_is_far_above_the_target(lx):
    """dX alone in bfloat16: words 20 to 41 above the target and 64 to 90 below another unit's, further apart than the powers of two of one number:
    each feeds a column of dX by itself."""
    T, d, V = 100, 64, 1024
    W, X = torch.zeros((V, d)), torch.zeros((T, d))
    X[:, 0] = 1 + torch.arange(T) % 5 / 128.0
    W[0, 0] = 105.0
    words = 384 + torch.arange(1, 64)
    W[words, 0] = 20.0 + torch.arange(1, 64) / 3.0
    W[words, torch.arange(1, 64)] = 1.0
    targets = torch.full((T,), V - 1, dtype=torch.int32)
    args = X.bfloat16().cuda(), W.bfloat16().cuda(), targets.cuda(), (0.5 + torch.arange(T) / T).cuda()
    out = call(lx, *args)
    check(*args, *out)
    dX, want = out[2].double().cpu()[:, 1:], ref.vocab_loss(args[0].cpu(), args[1].cpu(), targets, args[3].cpu())[2][:, 1:]
    # as in the test above, z up to 110; and what is below 2^-126 has bfloat16's smallest step, 2^-133
    limit = (2 * 2.0 ** -8 + 2.0 ** -16 + 4 * 110 * U + 300 * U) * want.abs() + 2 * 2.0 ** -133
    assert bool(((dX - want).abs() <= limit).all()), float(((dX - want).abs() / want.abs()).max()) * 2 ** 8
    assert float(want.abs().max()) > 1e-29 and bool((dX[want.abs() > 1e-37] != 0).all())
