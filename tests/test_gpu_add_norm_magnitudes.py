"""Norms of rows of values up to 1e18, whatever their length: the squares' sum is past fp32's largest, their mean is not."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("K", [64, 300, 1000, 1024, 2048, 4096, 4104, 8192, 16384, 17000, 300001])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("post", [False, True])
def test_large_values(dtype, rdtype, K, kind, post):
    rng = np.random.default_rng(K)
    P = 3
    low = 0.1 if kind == "rms" else -1.0
    make = lambda t: torch.from_numpy((0.5e18 * rng.uniform(low, 0.99, (P, K))).astype(np.float32)).to(R.TYPES[t])  # noqa: E731
    x, r = make(dtype), make(rdtype)
    n = (None, None, kind, float(np.float32(1e-5)))
    norm = fgq.Norm(kind=kind, eps=1e-5)
    s, y = fgq.fgq_add_norm(x.to(dev()), r.to(dev()), norm, post=norm if post else None)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want = R.add_norm(x.double().numpy(), r.double().numpy(), n, n if post else None, None, P, 1.0, dtype, rdtype)
    R.check(s.double().cpu().numpy(), *want[0], "residual")
    R.check(y.double().cpu().numpy(), *want[1], "y")


@pytest.mark.parametrize("K", [4096, 17000])
def test_equal_values(K):
    x = torch.full((2, K), 1e18, device=dev())
    assert torch.allclose(fgq.fgq_add_norm(x, None, fgq.Norm())[1], torch.ones_like(x), rtol=100 * 2.0 ** -24, atol=0)
    x = x.to(torch.bfloat16)
    assert torch.equal(fgq.fgq_add_norm(x, None, fgq.Norm())[1], torch.ones_like(x))
