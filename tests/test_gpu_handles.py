"""Norms and 4-bit weights as handles: what they are made of cannot be assigned, and a call takes their tensors as they are then."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def test_nothing_is_assigned():
    n = fgq.Norm(torch.ones(64, device=dev()), kind="layer", eps=1e-3)
    for name, value in (("weight", torch.zeros(64, device=dev())), ("bias", None), ("eps", 1.0), ("kind", "rms")):
        before = getattr(n, name)
        with pytest.raises(AttributeError):
            setattr(n, name, value)
        assert getattr(n, name) is before
    w = fgq.fgq_quantize_weights_w4(torch.ones((3, 20, 200), device=dev()), 32)
    assert (w.experts, w.rows, w.cols, w.group, w.codes.shape[0], w.scales.shape[0]) == (3, 20, 200, 32, 3, 3)
    for name in ("codes", "scales", "experts", "rows", "cols", "group"):
        with pytest.raises(AttributeError):
            setattr(w, name, getattr(w, name))


def test_norm_of_other_storage():
    rng = np.random.default_rng(0)
    x = R.rng_tensor(rng, (3, 64), "f32")[0].to(dev())
    make = lambda: R.rng_tensor(rng, (64,), "f32")[0].to(dev())  # noqa: E731
    w, b = make(), make()
    n = fgq.Norm(w, b, kind="layer")
    fgq.fgq_add_norm(x, None, n)
    for t in (w, b):
        t.data = make()
        assert torch.equal(fgq.fgq_add_norm(x, None, n, post=n)[1], fgq.fgq_add_norm(x, None, fgq.Norm(w.clone(), b.clone(), kind="layer"),
                                                                                      post=fgq.Norm(w.clone(), b.clone(), kind="layer"))[1])
    w.mul_(2)  # values may change in place
    assert torch.equal(fgq.fgq_add_norm(x, None, n)[1], fgq.fgq_add_norm(x, None, fgq.Norm(w.clone(), b, kind="layer"))[1])
    w.data = make()[:32].clone()
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, None, n)
    w.data = make().half()
    with pytest.raises(TypeError):
        fgq.fgq_add_norm(x, None, n)


def test_weights_of_other_storage():
    rng = np.random.default_rng(1)
    make = lambda e=(4,): fgq.fgq_quantize_weights_w4(R.rng_tensor(rng, e + (64, 64), "f32")[0].to(dev()), 32)  # noqa: E731
    g, u, d = make(), make(), make()
    x = R.rng_tensor(rng, (3, 64), "bf16")[0].to(dev())
    r = R.rng_tensor(rng, (4, 64), "bf16")[0].to(dev())
    fgq.fgq_moe_w4(x, r, 2, g, u, d)
    for w in (g, u, d):
        other = make()
        w.codes.data, w.scales.data = other.codes.clone(), other.scales.clone()
        assert torch.equal(fgq.fgq_read_weights_w4(w), fgq.fgq_read_weights_w4(other))
    fresh = [fgq.W4Weights(w.codes.clone(), w.scales.clone(), 64, 64) for w in (g, u, d)]
    assert torch.equal(fgq.fgq_moe_w4(x, r, 2, g, u, d), fgq.fgq_moe_w4(x, r, 2, *fresh))
    other = make((9,))
    g.codes.data, g.scales.data = other.codes.clone(), other.scales.clone()
    with pytest.raises(ValueError):
        fgq.fgq_moe_w4(x, r, 2, g, u, d)
    one = make(())
    one.codes.data = make((2,)).codes.clone()
    with pytest.raises(ValueError):
        fgq.fgq_linear_w4(x, one)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
