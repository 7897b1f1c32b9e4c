"""Routing with so little to multiply that a cluster's blocks reach their first keys at once: every key arrives."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("K,E,top", [(1, 3, 2), (8, 1, 1), (8, 8, 3), (40, 17, 4), (8, 300, 5)])
def test_short_rows(dtype, K, E, top):
    """More clusters than run at once, so that blocks begin at any time beside others that end."""
    rng = np.random.default_rng(K + E)
    P = 9001
    # logits are multiples of 1 / 64, exact in fp32: equal ones are ties
    x = torch.from_numpy(rng.choice([-2.0, -1.0, 1.0, 2.0], (P, K)).astype(np.float32)).to(R.TYPES[dtype])
    r = torch.from_numpy(rng.integers(-9, 10, (E, K)).astype(np.float32) / 64).to(R.TYPES[dtype])
    want, g, e = R.route(x.double().numpy(), r.double().numpy(), top, "softmax", True, 1.0)
    x, r = x.to(dev()), r.to(dev())
    for _ in range(20):
        ids, w = fgq.fgq_route_tokens(x, r, top)
        assert np.array_equal(ids.cpu().numpy(), want)
        R.check(w.double().cpu().numpy(), g, e * g, "weights")
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
