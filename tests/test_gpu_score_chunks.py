"""Some dozen to some hundred queries over a long cache (a prompt in chunks), either side of the number of queries from which calls go by
rows, forward and backward."""
import math

import pytest
import torch

from test_gpu_score_attn import Call, lx  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "f16")])
@pytest.mark.parametrize("Sq", [16, 17, 64, 128, 129])
def test_chunks(lx, Sq, D, dtype):  # noqa: F811
    lengths = [5000, Sq, 2049]
    c = Call(lx, 3, 4, 2, Sq, 5000, D, dtype, seed=70 + Sq, cap=(0.0, 8.0)[Sq % 2], slopes=Sq == 64, q_start=torch.tensor(lengths) - Sq)
    for b, n in enumerate(lengths):       # behind a sequence's end
        for t in (c.K, c.V):
            t[b, :, n:] = (math.nan, math.inf, -math.inf)[b]
    c.check()
    for b, n in enumerate(lengths):
        assert not c.dK[b, :, n:].any() and not c.dV[b, :, n:].any()
