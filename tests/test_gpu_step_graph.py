"""The calls of a decoding step and of a training step in captured graphs, replayed with other inputs and eager work between."""
import pytest
import torch

from test_gpu_score_attn import lx, tensor  # noqa: F401  (lx: a fixture)

pytestmark = pytest.mark.gpu


def replayed(step, change, outputs):
    """step() captured, then replays against eager runs of the same inputs, bit for bit."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        change(i)
        for t in outputs:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, outputs):
            assert not torch.isnan(a.float()).any() and torch.equal(a, b), i


@pytest.mark.parametrize("C", [600, 5000])          # whole pairs, equal runs
def test_decoding(lx, C):  # noqa: F811
    g = torch.Generator().manual_seed(3)
    Q, K = tensor(g, 3, 8, 1, 64, "bf16"), tensor(g, 3, 2, 1, 64, "bf16")
    cache_k, cache_v = tensor(g, 3, 2, C, 64, "bf16", "bhsd"), tensor(g, 3, 2, C, 64, "bf16", "bhsd")
    table, at = lx.lx_rope_table(64, C), torch.zeros(3, dtype=torch.int32, device="cuda")
    Qt, Kt, O, LSE = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(Q), torch.empty((3, 8, 1), device="cuda")

    def step():
        lx.lx_rope(Q, K, table, at.view(3, 1), Qt, Kt)
        cache_k.scatter_(2, at.long().view(3, 1, 1, 1).expand(3, 2, 1, 64), Kt)
        lx.lx_score_attn_fwd(Qt, cache_k, cache_v, 0.125, True, O, LSE, q_start=at)

    def change(i):
        at.copy_(torch.tensor([i, C // 2 + i, C - 1 - i], dtype=torch.int32))
        Q.mul_(1.25)
    replayed(step, change, [O, LSE])


def test_training(lx):  # noqa: F811
    g = torch.Generator().manual_seed(4)
    Q, K, V, dO = (tensor(g, 2, h, 200, 64, "f16", "bhsd") for h in (4, 2, 2, 4))
    begin, end = torch.tensor([0, 90, 200], dtype=torch.int32, device="cuda"), torch.tensor([90, 180, 400], dtype=torch.int32, device="cuda")
    lo, hi = (torch.empty((2, 200), dtype=torch.int32, device="cuda") for _ in range(2))
    O, dQ, dK, dV, LSE = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V), torch.empty((2, 4, 200), device="cuda")
    small, norm = torch.zeros(77, device="cuda"), torch.zeros(1, device="cuda")
    grads = lx.GradSet([dV, small], [dV, small])

    def step():
        lx.lx_attn_key_ranges(begin, end, None, True, lo, hi)
        lx.lx_score_attn_fwd(Q, K, V, 0.125, True, O, LSE, key_lo=lo, key_hi=hi)
        lx.lx_score_attn_bwd(Q, K, V, O, LSE, dO, 0.125, True, dQ, dK, dV, key_lo=lo, key_hi=hi)
        small.copy_(dQ.view(-1)[:77])
        lx.lx_grad_norm_clip(grads, 0.5, norm)

    def change(i):
        end[1] = 100 + 10 * i
        dO.mul_(0.5)
    # (padding: queries 100 + 10 i .. 199 of the first row attend nothing, whose LSE is -inf)
    replayed(step, change, [O, dQ, dK, dV, norm])
