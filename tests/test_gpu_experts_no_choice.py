"""Experts' calls of several passes of which some have no choice that is an expert: nothing of one pass reaches into the next."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_moe_w4 import layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("top,none", [(1, (0,)), (1, (0, 1)), (2, (0, 2)), (2, (1,)), (1, (0, 1, 2))])
def test_passes_without_choices(dtype, top, none):
    """Passes of 4096 choices, few enough an expert to hold a unit's tokens in shared memory; `none`: passes of which no choice is an expert."""
    rng = np.random.default_rng(top + len(none))
    E, K, F, per = 700, 72, 24, 4096 // top
    P = 2 * per + 57
    on, d = layer(rng, E, K, F, 32)
    x, x64 = R.rng_tensor(rng, (P, K), dtype)
    ids = rng.integers(0, E, (P, top)).astype(np.int32)
    for n in none:
        ids[n * per:(n + 1) * per] = rng.choice([-1, E, 2 ** 31 - 1], ids[n * per:(n + 1) * per].shape)
    g = rng.random((P, top)).astype(np.float32)
    xd, i, w = x.to(dev()), torch.from_numpy(ids).to(dev()), torch.from_numpy(g).to(dev())
    first = fgq.fgq_experts_w4(xd, i, w, *on)
    for _ in range(20):  # each frees its temporaries behind kernels under way, and the next takes them
        assert torch.equal(fgq.fgq_experts_w4(xd, i, w, *on), first)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.experts(x64, ids, g.astype(np.float64), np.zeros((P, 1)), *d, 32, 32, dtype)
    R.check(first.double().cpu().numpy(), want, bound, "passes")
