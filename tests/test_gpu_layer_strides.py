"""Outputs in memory of their own: axes in either order, gaps, single tokens with any stride; overlapping ones are refused."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def test_rope_strides():
    rng = np.random.default_rng(0)
    B, T, H, D = 3, 5, 2, 16
    x = R.rng_tensor(rng, (B, T, H, D), "bf16")[0].to(dev())
    table, starts = fgq.rope_table(D, device=dev()), torch.tensor([3, 70, 9], dtype=torch.int32, device=dev())
    want = fgq.fgq_rope(x, table, starts)
    big = torch.empty((T, B, H + 1, D), dtype=x.dtype, device=dev())
    for out in (big[:, :, :H].transpose(0, 1), torch.empty((T, B, H, D), dtype=x.dtype, device=dev()).transpose(0, 1),
                torch.empty((B, T + 2, H + 3, D), dtype=x.dtype, device=dev())[:, 1:T + 1, 2:H + 2]):
        assert torch.equal(fgq.fgq_rope(x, table, starts, out=out), want)
        out.copy_(x)
        assert torch.equal(fgq.fgq_rope(out, table, starts, out=out), want)
    one = torch.empty((1, 1, H, D), dtype=x.dtype, device=dev())
    assert torch.equal(fgq.fgq_rope(x[:1, :1], table, starts[:1], out=one.expand(1, 1, H, D)), want[:1, :1])
    for out in (torch.empty((B, 1, H, D), dtype=x.dtype, device=dev()).expand(B, T, H, D), torch.empty((1, T, H, D), dtype=x.dtype, device=dev()).expand(B, T, H, D)):
        with pytest.raises(fgq.FGQError) as e:
            fgq.fgq_rope(x, table, starts, out=out)
        assert e.value.code == fgq.FGQ_ERR_ARG


def test_norm_strides():
    rng = np.random.default_rng(1)
    x = R.rng_tensor(rng, (4, 24), "f32")[0].to(dev())
    n = fgq.Norm()
    s, y = fgq.fgq_add_norm(x[:, :16], x[:, 8:], n)
    with pytest.raises(fgq.FGQError):  # rows of y across rows of x
        fgq.fgq_add_norm(x[:, :16], None, n, y=x.view(-1)[:64].view(4, 16))
    r = x.clone()
    with pytest.raises(fgq.FGQError):
        fgq.fgq_add_norm(x[:, :16], r[:, :16], n, residual_out=r.view(-1)[:64].view(4, 16))
    r = x.clone()
    s2, y2 = fgq.fgq_add_norm(x[:, :16], r[:, 8:], n, residual_out=r[:, 8:])  # another view of the same rows
    assert torch.equal(r[:, 8:], s) and torch.equal(y2, y)
    r = x[:1, :16].clone()
    assert torch.equal(fgq.fgq_add_norm(r, None, n, y=r)[1], fgq.fgq_add_norm(x[:1, :16], None, n)[1])
