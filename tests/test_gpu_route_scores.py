"""Routers' scores far from 1."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_moe_w4 import layer

pytestmark = pytest.mark.gpu

LOGITS = {"all one": [-100.0] * 6, "border": [-87.0, -87.5, -88.25, -88.75, -89.0, -90.0], "far": [-200.0, -201.0, -203.5, -260.0, -205.0, -200.25],
          "mixed": [-3.0, -90.0, -120.0, 2.0, -89.0, -0.5], "one high": [-95.0, -96.0, 40.0, -97.0, -300.0, -95.0], "high": [90.0, 100.0, 200.0, 95.0, 150.0, 90.5],
          "lowest": [-600.0, -601.0, -602.0, -600.5, -604.0, -599.0]}


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("P,top", [(1, 1), (3, 3), (9, 6)])
@pytest.mark.parametrize("which", list(LOGITS))
def test_sigmoid_scores(which, P, top, renormalize):
    """Finite weights of finite logits: a ratio of scores that fp32 does not hold is held.  (Logits are exact in fp32, so their errors are none; scores
    below 2^-126 are rounded to multiples of 2^-149, as fp32 is.)"""
    l = np.array(LOGITS[which])
    x = torch.ones((P, 8), device=dev())
    r = torch.zeros((6, 8), device=dev())
    r[:, 2] = torch.from_numpy(l.astype(np.float32)).to(dev())
    ids, w = fgq.fgq_route_tokens(x, r, top, "sigmoid", renormalize, 1.5)
    want, g, e = R.route(np.ones((P, 8)), r.double().cpu().numpy(), top, "sigmoid", renormalize, 1.5)
    assert np.array_equal(ids.cpu().numpy(), want)
    R.check(w.double().cpu().numpy(), g, e * g + 2 * 2.0 ** -149, "weights")
    assert torch.isfinite(w).all()


@pytest.mark.parametrize("P", [1, 4, 40])
def test_outputs_of_low_scores(P):
    rng = np.random.default_rng(P)
    on, d = layer(rng, 6, 64, 32, 32)
    x = R.rng_tensor(rng, (P, 64), "bf16")[0]
    x[:, 0] = 1.0
    r = torch.zeros((6, 64))
    r[:, 0] = torch.tensor(LOGITS["far"])
    y = fgq.fgq_moe_w4(x.to(dev()), r.to(dev()), 3, *on, score="sigmoid")
    ids, g, e = R.route(x.double().numpy(), r.double().numpy(), 3, "sigmoid", True, 1.0)
    want, bound = R.experts(x.double().numpy(), ids, g, e, *d, 32, 32, "bf16")
    R.check(y.double().cpu().numpy(), want, bound, "layer")
