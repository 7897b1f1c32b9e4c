"""Routing of tokens that hold infinities."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,E", [(1, 16, 9), (6, 1000, 40), (5, 13, 130)])
def test_infinite_tokens(dtype, P, K, E):
    """A token with an infinity: infinite logits, the largest first, equal ones by their index; sigmoid scores 1 and 0, softmax NaN; other tokens as
    without it."""
    rng = np.random.default_rng(K)
    x = R.rng_tensor(rng, (P, K), dtype)[0].to(dev())
    r = R.rng_tensor(rng, (E, K), dtype)[0].to(dev())
    at = K - 2
    sign = torch.ones(E)
    sign[[2, 5, E - 1]] = -1.0
    r[:, at] = (sign * 0.5).to(r.dtype).to(dev())
    before = fgq.fgq_route_tokens(x, r, 5, "sigmoid", True)
    p = P // 2
    x[p, at] = -float("inf")
    logits = x.double().cpu() @ r.double().cpu().t()
    assert torch.isinf(logits[p]).all()
    want = [2, 5, E - 1, 0, 1]
    keep = [i for i in range(P) if i != p]
    for renormalize, w in ((True, 1 / 3), (False, 1.0)):
        ids, g = fgq.fgq_route_tokens(x, r, 5, "sigmoid", renormalize)
        assert ids[p].tolist() == want
        assert torch.equal(g[p].cpu(), torch.tensor([w, w, w, 0.0, 0.0]))
        assert torch.equal(ids[keep], before[0][keep]) and (not renormalize or torch.equal(g[keep], before[1][keep]))
    ids, g = fgq.fgq_route_tokens(x, r, 5)
    assert ids[p].tolist() == want and torch.isnan(g[p]).all() and torch.isfinite(g[keep]).all()
    x[p, at] = float("inf")
    assert fgq.fgq_route_tokens(x, r, 2)[0][p].tolist() == [0, 1]
