"""The calls between and behind a layer's halves, without a GPU: what the C entry points refuse before any launch, what reaches them
through the binding, the generator's published vectors, and the definitions' gradients against differences."""
import ctypes as C
import math

import pytest
import torch

import block_reference as ref

P = 0x1000      # non-null, 16-byte aligned, never dereferenced on these paths


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def strides(*s):
    return (C.c_int64 * len(s))(*s)


# --- refusals ---------------------------------------------------------------------------------

ROWS_BAD = (dict(T=0), dict(d=0), dict(T=-1), dict(d=-8), dict(X=None), dict(X=P + 1), dict(st=None))
DROP_BAD = (dict(p=-0.1), dict(p=1.0), dict(p=math.nan), dict(p=0.999999), dict(p=0.1, rng=None), dict(p=0.1, rng=P + 4))


def dropout(lx, **kw):
    c = {**dict(dt=1, T=8, d=64, X=P, R=P, out=P, st=(64, 64, 64), p=0.1, rng=P, site=0), **kw}
    st = None if c["st"] is None else strides(*c["st"])
    return lx._lib.lx_dropout(c["dt"], c["T"], c["d"], c["X"], c["R"], c["out"], st, c["p"], c["rng"], c["site"], None)


def test_dropout_refuses(lx):
    for bad in ROWS_BAD + DROP_BAD + (dict(out=None), dict(R=P + 1), dict(out=P + 1), dict(st=(-1, 64, 64)), dict(st=(64, -1, 64)), dict(st=(64, 64, 63))):
        assert dropout(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    assert dropout(lx, dt=5) == lx.LX_ERR_UNSUPPORTED


def norm_fwd(lx, **kw):
    c = {**dict(dt=1, T=8, d=256, eps=1e-5, w=P, X=P, R=P, H=P, Y=P, st=(256, 256, 256, 256), Y8=None, scales=None, group=0, p=0.0, rng=P), **kw}
    st = None if c["st"] is None else strides(*c["st"])
    return lx._lib.lx_rms_norm_fwd(c["dt"], c["T"], c["d"], c["eps"], c["w"], c["X"], c["R"], c["H"], c["Y"], st, c["Y8"], c["scales"], c["group"],
                                   c["p"], c["rng"], 0, None)


def test_norm_refuses(lx):
    for bad in ROWS_BAD + DROP_BAD + (
            dict(Y=None), dict(eps=-1e-5), dict(eps=math.nan), dict(eps=math.inf), dict(w=P + 1), dict(R=P + 1), dict(H=P + 1), dict(Y=P + 1),
            dict(st=(256, 256, 255, 256)), dict(st=(256, 256, 256, 255)), dict(st=(256, -256, 256, 256)), dict(Y8=P), dict(scales=P),
            dict(Y8=P, scales=P + 2, group=256), dict(Y8=P, scales=P, group=0), dict(Y8=P, scales=P, group=96), dict(Y8=P, scales=P, group=-32)):
        assert norm_fwd(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    wide = dict(d=32769, st=(32769,) * 4)
    assert norm_fwd(lx, dt=3) == norm_fwd(lx, **wide) == norm_fwd(lx, Y8=P, scales=P, group=16) == lx.LX_ERR_UNSUPPORTED


def norm_bwd(lx, **kw):
    c = {**dict(dt=1, T=8, d=256, eps=1e-5, w=P, X=P, H=P, dH=P, dX=P, dR=P, st=(256,) * 5, dW=P, p=0.0, rng=P, ws=P, bytes=1 << 30), **kw}
    st = None if c["st"] is None else strides(*c["st"])
    return lx._lib.lx_rms_norm_bwd(c["dt"], c["T"], c["d"], c["eps"], c["w"], c["X"], c["H"], c["dH"], c["dX"], c["dR"], st, c["dW"], c["p"], c["rng"],
                                   0, c["ws"], c["bytes"], None)


def test_norm_backward_refuses(lx):
    for bad in ROWS_BAD + DROP_BAD + (
            dict(H=None), dict(dX=None, dR=None, dW=None), dict(eps=-1.0), dict(H=P + 1), dict(dH=P + 1), dict(dX=P + 1), dict(dR=P + 1), dict(dW=P + 2),
            dict(st=(256, 256, 256, 8, 256)), dict(st=(256, 256, 256, 256, 8)), dict(st=(256, 256, -8, 256, 256)), dict(ws=P + 8)):
        assert norm_bwd(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    assert norm_bwd(lx, d=40000, st=(40000,) * 5) == lx.LX_ERR_UNSUPPORTED
    need = lx.lx_rms_norm_bwd_workspace_bytes(8, 256)
    assert need >= 256 * 4
    assert norm_bwd(lx, bytes=need - 1) == norm_bwd(lx, ws=None) == lx.LX_ERR_WORKSPACE
    assert lx.lx_rms_norm_bwd_workspace_bytes(0, 64) == lx.lx_rms_norm_bwd_workspace_bytes(8, 40000) == 0


def vocab_loss(lx, **kw):
    c = {**dict(dt=1, T=8, d=64, V=100, X=P, xs=64, W=P, targets=P, weights=P, loss=P, lse=P, dX=P, dxs=64, dW=P, dw=1, ws=P, bytes=1 << 40), **kw}
    return lx._lib.lx_vocab_loss(c["dt"], c["T"], c["d"], c["V"], c["X"], c["xs"], c["W"], c["targets"], c["weights"], c["loss"], c["lse"], c["dX"],
                                 c["dxs"], c["dW"], c["dw"], c["ws"], c["bytes"], None)


def test_vocab_loss_refuses(lx):
    for bad in (dict(T=0), dict(d=0), dict(V=0), dict(T=-3), dict(X=None), dict(W=None), dict(targets=None), dict(loss=None), dict(X=P + 1), dict(W=P + 8),
                dict(targets=P + 2), dict(weights=P + 2), dict(loss=P + 1), dict(lse=P + 2), dict(dX=P + 1), dict(dW=P + 8), dict(xs=-1), dict(dxs=63),
                dict(ws=P + 8)):
        assert vocab_loss(lx, **bad) == lx.LX_ERR_INVALID_ARG, bad
    for bad in (dict(dt=4), dict(d=96), dict(d=65536), dict(V=(1 << 20) + 1), dict(T=(1 << 31) - 1), dict(dw=2), dict(dw=5), dict(dt=0, dw=1)):
        assert vocab_loss(lx, **bad) == lx.LX_ERR_UNSUPPORTED, bad
    assert vocab_loss(lx, ws=None) == vocab_loss(lx, bytes=1000) == lx.LX_ERR_WORKSPACE


def test_vocab_loss_workspace(lx):
    f = lx.lx_vocab_loss_workspace_bytes
    both = lx.LX_GRAD_X | lx.LX_GRAD_W
    assert f(3, 8, 64, 100) == f(lx.LX_BF16, 0, 64, 100) == f(lx.LX_BF16, 8, 100, 100) == f(lx.LX_BF16, 8, 64, 100, tokens=-1) == 0
    sizes = [f(lx.LX_BF16, 8192, 2048, 50272, both, lx.LX_BF16, t) for t in (256, 512, 4096, 0)]
    assert sizes[0] < sizes[1] < sizes[2]
    need = f(lx.LX_BF16, 8192, 2048, 50272, both, lx.LX_BF16, 256)
    assert vocab_loss(lx, T=8192, d=2048, V=50272, xs=2048, dxs=2048, bytes=need - 1) == lx.LX_ERR_WORKSPACE
    # a piece's gradients stay within 1 GiB, whatever the call
    assert f(lx.LX_F32, 1 << 22, 512, 262144) < (1 << 31)
    assert f(lx.LX_BF16, 1 << 22, 512, 262144) < (1 << 31)
    assert f(lx.LX_BF16, 1 << 22, 512, 262144, 0) < (1 << 31)


# --- the binding ------------------------------------------------------------------------------

def test_binding_refuses_tensors_elsewhere(lx, monkeypatch):
    """Tensors on the host, of other sizes, types or layouts, before the library is called."""
    calls = lx._call
    x, w = torch.zeros((4, 64)), torch.zeros(64)
    device = torch.cuda.current_device() if torch.cuda.is_available() else None
    if device is not None:
        with pytest.raises(AssertionError):
            lx.lx_dropout(x, x, 0.0, None)
        return
    calls.bind_block({n: C.cast(getattr(lx._lib, n), C.c_void_p).value for n in lx.EXPORTS}, lambda: -1, torch.int64, torch.float8_e4m3fn)
    monkeypatch.setattr(lx, "_call", calls)
    try:
        for bad in (dict(out=x[:3]), dict(out=x.double()), dict(residual=x.t()), dict(out=torch.zeros((64, 4)).t()), dict(rng=torch.zeros(2)),
                    dict(rng=torch.zeros(3, dtype=torch.int64)), dict(X=x[0])):
            a = {**dict(X=x, out=x, rng=None, residual=None), **bad}
            with pytest.raises((AssertionError, ValueError)):
                lx.lx_dropout(a["X"], a["out"], 0.1, a["rng"], residual=a["residual"])
        y8, scales = torch.zeros((4, 64), dtype=torch.float8_e4m3fn), torch.zeros((4, 2))
        for bad in (dict(weight=w[:3]), dict(weight=w.half()), dict(Y8=y8, scales=scales[:, :1].double()), dict(Y8=y8, scales=torch.zeros((4, 5))),
                    dict(Y8=y8, scales=torch.zeros((3, 2))), dict(Y8=y8[:2], scales=scales), dict(Y8=torch.zeros((4, 64), dtype=torch.uint8), scales=scales),
                    dict(Y8=torch.zeros((64, 4), dtype=torch.float8_e4m3fn), scales=scales)):
            a = {**dict(weight=w, Y8=None, scales=None), **bad}
            with pytest.raises(AssertionError):
                lx.lx_rms_norm_fwd(x, a["weight"], 1e-5, x, Y8=a["Y8"], scales=a["scales"])
        for bad in (dict(H=None), dict(dX=x[:2]), dict(dW=w.half()), dict(dW=w[:5])):
            a = {**dict(H=x, dX=x, dW=None), **bad}
            with pytest.raises(AssertionError):
                lx.lx_rms_norm_bwd(x, a["H"], w, 1e-5, a["dX"], dW=a["dW"])
    finally:
        calls.bind_block({n: C.cast(getattr(lx._lib, n), C.c_void_p).value for n in lx.EXPORTS}, lx._device, torch.int64, torch.float8_e4m3fn)


# --- definitions ------------------------------------------------------------------------------

def test_generator_gives_the_published_numbers():
    assert ref.philox((0,) * 4, (0, 0)) == (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)
    assert ref.philox((ref.MASK,) * 4, (ref.MASK,) * 2) == (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)


def test_shares_of_dropped_elements():
    f = ref.factors(64, 100, 0.25, seed=3, step=1, site=2)
    kept = float((f != 0).double().mean())
    assert abs(kept - 0.75) < 5 * math.sqrt(0.25 * 0.75 / f.numel())
    assert not torch.equal(f, ref.factors(64, 100, 0.25, seed=3, step=2, site=2)) and not torch.equal(f, ref.factors(64, 100, 0.25, seed=3, step=1, site=1))


def test_vocab_loss_gradients_against_differences():
    g = torch.Generator().manual_seed(2)
    X, W = torch.randn((4, 6), generator=g, dtype=torch.float64), torch.randn((5, 6), generator=g, dtype=torch.float64)
    targets, weights = torch.tensor([2, -100, 0, 4]), torch.tensor([0.5, 2.0, -1.0, 3.0], dtype=torch.float64)

    def loss(X, W):
        return float((ref.vocab_loss(X, W, targets)[0] * weights).sum())
    _, _, dX, dW = ref.vocab_loss(X, W, targets, weights)
    for r in range(5):
        for c in range(6):
            assert abs(difference(lambda v: loss(X, v), W, (r, c)) - dW[r, c]) < 1e-7
            if r < 4:
                assert abs(difference(lambda v: loss(v, W), X, (r, c)) - dX[r, c]) < 1e-7


def difference(loss, x, at, h=1e-5):
    up, down = x.clone(), x.clone()
    up[at] += h
    down[at] -= h
    return (loss(up) - loss(down)) / (2 * h)


def test_norm_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    x, r, dy, dh = (torch.randn((3, 11), generator=g, dtype=torch.float64) for _ in range(4))
    w = torch.randn(11, generator=g, dtype=torch.float64)
    f = ref.factors(3, 11, 0.3, 5, 0, 0)

    def loss(x, r, w):
        h, y = ref.norm(x, r, w, 1e-2, f)
        return float((y * dy).sum() + (h * dh).sum())
    dX, dR, dW = ref.norm_back(dy, ref.norm(x, r, w, 1e-2, f)[0], w, 1e-2, dh, f)
    for t in range(3):
        for c in range(11):
            assert abs(difference(lambda v: loss(v, r, w), x, (t, c)) - dX[t, c]) < 1e-7
            assert abs(difference(lambda v: loss(x, v, w), r, (t, c)) - dR[t, c]) < 1e-7
    for c in range(11):
        assert abs(difference(lambda v: loss(x, r, v), w, c) - dW[c]) < 1e-7
