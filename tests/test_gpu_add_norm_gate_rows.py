"""Gates whose row stands for more tokens than there are: any number, also past 32 bits."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("per", [7, 8, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 32 + 3, 2 ** 40])
def test_one_row_for_all(per):
    rng = np.random.default_rng(0)
    x = R.rng_tensor(rng, (7, 64), "bf16")[0].to(dev())
    g = R.rng_tensor(rng, (1, 64), "bf16")[0].to(dev())
    n = fgq.Norm()
    want = fgq.fgq_add_norm(x, None, n, gate=g.expand(7, 64).contiguous(), tokens_per_gate=1)
    for gate in (g, g[0]):
        got = fgq.fgq_add_norm(x, None, n, gate=gate, tokens_per_gate=per)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
