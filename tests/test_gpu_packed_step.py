"""The example of a packed fine-tuning step: rotary positions, key ranges, attention, the LoRA FFN, clipping and the cache, run
together as a program would."""
import importlib.util
import os

import pytest
import torch

from util import FRO, rel_err_fro

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2510_15964_amd import build
    build.ensure()
    spec = importlib.util.spec_from_file_location("packed_step", os.path.join(ROOT, "examples", "packed_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("size", [dict(width=256, heads=4, kv_heads=4, ffn=512, rows=2, tokens=256),
                                  dict(width=512, heads=4, kv_heads=2, ffn=1024, rows=3, tokens=448)])
def test_packed_step(example, size):
    r = example.run(**size)
    for t in (r["out"], r["dx"], *r["raw"], *r["clipped"]):
        assert torch.isfinite(t).all()
    # a document gets the same attention in a pack as alone, and its last token the same from the cache: sums in another order,
    # so a rounding of P and one of O apart
    fro = 2 * FRO["bf16"]
    assert rel_err_fro(r["packed"].float().cpu().numpy(), r["alone"].double().cpu().numpy()) <= fro
    assert rel_err_fro(r["token"].float().cpu().numpy(), r["alone"][:, :, -1:].double().cpu().numpy()) <= fro
    # the norm, in 64 bits, to the rounding of its one number to fp32; the gradients scaled by a factor and a product rounded once
    norm = sum(t.double().square().sum() for t in r["raw"]).sqrt().item()
    assert norm > r["max_norm"] and abs(r["norm"] - norm) <= norm * 2.0 ** -23
    for raw, cut in zip(r["raw"], r["clipped"]):
        want = raw.double() * (r["max_norm"] / norm)
        assert (cut.double() - want).abs().le(want.abs() * 2.0 ** -22 + 2.0 ** -149).all()
    # padding attends nothing and no loss comes from it: its gradient is zero
    assert (r["dx"][r["padding"]] == 0).all()


def test_pack(example):
    rows, begin, end = example.pack([5, 4, 3, 6, 1], 8)
    assert rows == 3 and begin == [0, 8, 5, 16, 12] and end == [5, 12, 8, 22, 13]
