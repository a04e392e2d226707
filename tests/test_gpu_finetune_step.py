"""Dropout, norm with residual and the loss over a vocabulary in a run: chained by themselves, and in the fine-tuning step of
examples/finetune_step.py, forward and backward against plain operations in 64 bits.

A call's result is off by the gates of util.py (FRO) at most, relative to its norm; of a chain of n calls, each of which passes on what
reaches it, by n of those."""
import math
import os
import sys

import pytest
import torch

import block_reference as ref
from util import FRO, torch_dtype

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def far(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


def normed(h, w, eps):
    return h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * w


def mean_loss(y, W, targets, weights):
    held = (targets >= 0) & (targets < W.shape[0])
    z = torch.log_softmax(y[held] @ W.t(), -1)
    return -(z.gather(1, targets[held].long()[:, None])[:, 0] * weights[held]).sum()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_chain(lx, dtype):
    """x -> dropout -> h = r + . -> norm -> linear -> h' = h + dropout(.) -> norm -> loss, and back."""
    T, d, V, eps, p = 70, 128, 301, 1e-5, 0.2
    g = torch.Generator().manual_seed(1)
    dt = torch_dtype(dtype)
    x, r, M, W = (t.to(dt) for t in (torch.randn((T, d), generator=g), torch.randn((T, d), generator=g), torch.randn((d, d), generator=g) * d ** -0.5,
                                     torch.randn((V, d), generator=g) * 2 * d ** -0.5))
    w1, w2 = ((1 + 0.2 * torch.randn(d, generator=g)).to(dt) for _ in range(2))
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    targets[::3] = -100
    weights = torch.rand(T, generator=g) * (64 if dtype == "f16" else 1)
    cx, cr, cM, cW, c1, c2, ct, cw = (t.cuda() for t in (x, r, M, W, w1, w2, targets, weights))
    rng = torch.tensor([11, 3], dtype=torch.int64, device="cuda")
    h1, y1, h2, y2, dy2, dh2, dz, dx, dr = (torch.empty_like(cx) for _ in range(9))
    loss, dw1, dw2, dW = torch.empty(T, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty_like(cW)
    lx.lx_rms_norm_fwd(cx, c1, eps, y1, residual=cr, H=h1, p=p, rng=rng, site=1)
    z = y1 @ cM.t()
    lx.lx_rms_norm_fwd(z, c2, eps, y2, residual=h1, H=h2, p=p, rng=rng, site=2)
    lx.lx_vocab_loss(y2, cW, ct, loss, weights=cw, dX=dy2, dW=dW)
    lx.lx_rms_norm_bwd(dy2, h2, c2, eps, dz, dR=dh2, dW=dw2, p=p, rng=rng, site=2)
    dy1 = dz @ cM
    lx.lx_rms_norm_bwd(dy1, h1, c1, eps, dx, dH=dh2, dR=dr, dW=dw1, p=p, rng=rng, site=1)

    leaves = [t.double().requires_grad_() for t in (x, r, w1, w2, W)]
    X, R, A, B, Vm = leaves
    f1, f2 = ref.factors(T, d, p, 11, 3, 1), ref.factors(T, d, p, 11, 3, 2)
    a = R + X * f1
    b = a + (normed(a, A, eps) @ M.double().t()) * f2
    total = mean_loss(normed(b, B, eps), Vm, targets, weights.double())
    total.backward()
    total = float(total.detach())
    assert abs(float((loss * cw).sum()) - total) <= 5 * FRO[dtype] * total
    for got, leaf, calls in ((dx, X, 9), (dr, R, 9), (dw1, A, 9), (dw2, B, 7), (dW, Vm, 6)):
        assert far(got, leaf.grad) <= calls * FRO[dtype], (calls, far(got, leaf.grad))


def attention(Q, K, V, lo, hi, scale, cap):
    """[B,H,S,D] in 64 bits, one key interval per query; key heads shared."""
    S = Q.shape[2]
    K, V = (t.repeat_interleave(Q.shape[1] // t.shape[1], 1) for t in (K, V))
    z = cap * torch.tanh(Q @ K.transpose(-1, -2) * scale / cap)
    k = torch.arange(S)
    seen = (k >= lo[:, :, None]) & (k < hi[:, :, None]) & (k <= torch.arange(S)[:, None])
    some = seen.any(-1)
    z = z.masked_fill(~(seen | ~some[:, :, None])[:, None], -math.inf)
    return torch.softmax(z, -1) @ V * some[:, None, :, None]


def turned(x, table, positions):
    """Pairs i, i + D / 2 of [B,H,S,D] turned."""
    h = x.shape[-1] // 2
    c, s = table[positions][:, None, :, :h], table[positions][:, None, :, h:]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * c - b * s, a * s + b * c], -1)


def test_step(lx):
    import finetune_step
    r = finetune_step.run(width=256, heads=4, kv_heads=2, ffn=512, vocabulary=777, rows=2, tokens=128, p=0.1, max_norm=1e-3, active=1.0)
    L = r["layer"]
    x, lo, hi, pos, targets = (r[k].cpu() for k in ("x", "lo", "hi", "positions", "targets"))
    B, S, d = x.shape
    T = B * S
    f = [ref.factors(T, d, 0.1, 0, 0, site) for site in (1, 2)]
    cpu = lambda t: t.detach().double().cpu()  # noqa: E731
    leaves = [cpu(t).requires_grad_() for t in (x, L.A, L.B, *L.norms)]
    X, A, Bm, n0, n1, n2 = leaves
    Wqkv, Wo, Wu, Wd, Wv, table = (cpu(t) for t in (L.Wqkv, L.Wo, L.W_up, L.W_down, L.W_vocab, L.table))
    flat = X.view(T, d)
    qkv = (normed(flat, n0, finetune_step.EPS) @ Wqkv.t()).view(B, S, -1, L.D).transpose(1, 2)
    Q, K, V = qkv[:, :L.Hq], qkv[:, L.Hq:L.Hq + L.Hkv], qkv[:, L.Hq + L.Hkv:]
    O = attention(turned(Q, table, pos.long()), turned(K, table, pos.long()), V, lo, hi, L.D ** -0.5, finetune_step.CAP)
    h = flat + (O.transpose(1, 2).reshape(T, d) @ Wo.t()) * f[0]
    y = normed(h, n1, finetune_step.EPS)
    h = h + (torch.relu(y @ Wu.t() + (y @ A.t()) @ Bm.t()) @ Wd.t()) * f[1]
    total = mean_loss(normed(h, n2, finetune_step.EPS), Wv, targets, r["weights"].double().cpu())
    total.backward()
    total = float(total.detach())
    assert r["answers"] == int((targets >= 0).sum()) > 50 and bool((r["loss"][r["targets"] < 0] == 0).all())
    assert abs(float((r["loss"] * r["weights"]).sum()) - total) <= 8 * FRO["bf16"] * total
    # forward and back: 3 norms, projections, rotation, attention, two products of the FFN, loss, and their gradients
    wants = [X.grad, A.grad[:64], Bm.grad[:, :64], n0.grad, n1.grad, n2.grad]
    for got, want, calls in zip([r["dx"], *r["raw"]], wants, (20, 14, 14, 20, 16, 11)):
        assert far(got, want) <= calls * FRO["bf16"], (calls, far(got, want))
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in r["raw"]))
    assert abs(r["norm"] - norm) <= 2.0 ** -22 * norm and norm > r["max_norm"]
    for got, raw in zip(r["clipped"], r["raw"]):
        assert torch.allclose(got.double(), raw.double() * (r["max_norm"] / norm), rtol=2.0 ** -21, atol=0)


def test_step_at_its_defaults_and_replayed(lx):
    """The example at a larger size, and two steps whose masks differ by the step alone."""
    import finetune_step
    r = finetune_step.run(width=512, heads=8, kv_heads=2, ffn=1024, vocabulary=5003, rows=2, tokens=256)
    L = r["layer"]
    blocks = lx.lx_mask_compact(r["mask"])
    args = (r["x"], r["positions"], r["lo"], r["hi"], blocks, r["targets"], r["weights"])
    assert int(L.rng[1]) == 1
    again, _ = L.step(*args)
    assert int(L.rng[1]) == 2 and not torch.equal(again, r["loss"])
    L.rng[1] = 0
    first, dx = L.step(*args)
    assert torch.equal(first, r["loss"]) and torch.equal(dx, r["dx"])


def test_captured_step(lx):
    """The whole step captured into a graph, replayed with other seeds and steps of the dropout and other inputs, with eager steps in between:
    loss, the gradient of x and all gradients into the layer's buffers bit by bit as the eager step's."""
    import finetune_step
    r = finetune_step.run(width=256, heads=4, kv_heads=2, ffn=512, vocabulary=1003, rows=2, tokens=128, p=0.2)
    L = r["layer"]
    held = [L.dA, L.dB, *L.dnorms]
    args = (r["x"], r["positions"], r["lo"], r["hi"], lx.lx_mask_compact(r["mask"]), r["targets"], r["weights"])

    def eager(rng):
        L.rng.copy_(rng)
        for t in held:
            t.fill_(math.nan)
        loss, dx = L.step(*args)
        assert L.rng.tolist() == [int(rng[0]), int(rng[1]) + 1]
        return [t.clone() for t in (loss, dx, *held)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.step(*args)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, dx = L.step(*args)
    seen = []
    for seed, step in ((0, 0), (0, 1), (5, 1), (0, 0)):
        rng = torch.tensor([seed, step], dtype=torch.int64)
        want = eager(rng)
        L.rng.copy_(rng)
        for t in (loss, dx, *held):
            t.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert L.rng.tolist() == [seed, step + 1]
        assert all(torch.equal(a, b) for a, b in zip((loss, dx, *held), want)), (seed, step)
        graph.replay()                               # the next step, its masks from the device's counter
        torch.cuda.synchronize()
        after = [t.clone() for t in (loss, dx, *held)]
        assert all(torch.equal(a, b) for a, b in zip(after, eager(rng + torch.tensor([0, 1]))))
        seen.append(want)
    assert all(torch.equal(a, b) for a, b in zip(seen[0], seen[3])) and not torch.equal(seen[0][0], seen[1][0]) and not torch.equal(seen[1][0], seen[2][0])
    r["x"].mul_(1.25)
    want = eager(torch.tensor([3, 4]))
    L.rng.copy_(torch.tensor([3, 4]))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((loss, dx, *held), want))
