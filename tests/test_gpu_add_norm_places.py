"""Outputs in their inputs' places, of every form, many rows at once."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("P,K", [(700, 512), (1, 1024), (700, 1024), (40, 2048), (700, 2048), (700, 2056), (40, 4096), (700, 4096), (701, 4095), (330, 8192), (330, 16384),
                                 (40, 17000)])
def test_in_place(dtype, rdtype, P, K):
    rng = np.random.default_rng(K)
    x = R.rng_tensor(rng, (P, K), dtype)[0].to(dev())
    r = R.rng_tensor(rng, (P, K), rdtype)[0].to(dev())
    g = R.rng_tensor(rng, (P, K), dtype)[0].to(dev())
    n = fgq.Norm(torch.rand(K, device=dev()), torch.rand(K, device=dev()), kind="layer")
    s, y = fgq.fgq_add_norm(x, r, n, post=n, gate=g, tokens_per_gate=1, scale=0.5)
    for both in (True, False):
        x1, r1 = x.clone(), r.clone()
        s1, y1 = fgq.fgq_add_norm(x1, r1, n, post=n, gate=g, tokens_per_gate=1, scale=0.5, residual_out=r1, y=x1 if both else None)
        assert s1 is r1 and torch.equal(s1, s) and torch.equal(y1, y)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
