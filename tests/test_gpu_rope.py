"""Rotary positions against the definition in 64 bits: both layouts, parts of a head, strides, far positions, ragged batches."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def run(rng, B, T, heads, D, rot, dtype, layout="half", starts=None, lens=None, magnitude=1.0, inverse=False, view=0, in_place=False,
        **table):
    """view: heads beside those that turn, in the same rows."""
    t, x = R.rng_tensor(rng, (B, T, heads + view, D), dtype)
    t = t.to(dev())
    before = t.clone()
    starts = rng.integers(0, 131072, B) if starts is None else starts
    f = R.freqs(rot, **table)
    tab = fgq.rope_table(rot, device=dev(), **table)
    st = torch.tensor(np.asarray(starts), dtype=torch.int32, device=dev())
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev())
    part = t[:, :, view // 2:view // 2 + heads]
    y = fgq.fgq_rope(part, tab, st, lens=ln, layout=layout, magnitude=magnitude, inverse=inverse, out=part if in_place else None)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.rope(x[:, :, view // 2:view // 2 + heads], f, starts, lens, layout, np.float32(magnitude), inverse, dtype)
    R.check(y.double().cpu().numpy(), want, bound, "rope")
    if in_place:
        t[:, :, view // 2:view // 2 + heads] = before[:, :, view // 2:view // 2 + heads]
    assert torch.equal(t, before)  # nothing else was written


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("B,T,heads,D,rot", [(1, 1, 1, 2, 2), (3, 1, 5, 64, 64), (2, 7, 40, 128, 128), (2, 33, 3, 80, 20), (1, 70, 2, 96, 48),
                                             (5, 4, 1, 256, 64), (2, 9, 3, 7, 6), (1, 300, 12, 128, 32)])
@pytest.mark.parametrize("in_place", [False, True])
def test_shapes(dtype, layout, B, T, heads, D, rot, in_place):
    rng = np.random.default_rng(B * T + D)
    run(rng, B, T, heads, D, rot, dtype, layout, view=2, in_place=in_place)


@pytest.mark.parametrize("lens", [[0, 5, 9], [9, 1, 12], [-3, 0, 0]])
@pytest.mark.parametrize("in_place", [False, True])
def test_ragged(lens, in_place):
    rng = np.random.default_rng(1)
    for layout in ("half", "interleaved"):
        run(rng, 3, 9, 4, 64, 32, "bf16", layout, lens=lens, in_place=in_place)


@pytest.mark.parametrize("starts", [[0, -1], [-5, -100000], [2 ** 31 - 1, 2 ** 31 - 3], [-2 ** 31, 2 ** 30]])
def test_far_positions(starts):
    """Past the largest int32 as well.  64-bit angles are off by 2^31 2^-53 radians at most, the table by 2^31 2^-65 turns."""
    run(np.random.default_rng(2), 2, 6, 2, 128, 128, "f32", starts=starts)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="ramp", factor=8.0, length=4096.0), dict(base=5e5, scaling="ramp", factor=2.0, length=8192.0, high=4.0)])
def test_scaled(kw):
    run(np.random.default_rng(3), 2, 5, 3, 128, 128, "f32", magnitude=1.2079, **kw)


def test_there_and_back():
    """The inverse gives x back; and it is the gradient: (J^T g).x = g.(J x) for the linear map J."""
    rng = np.random.default_rng(4)
    tab = fgq.rope_table(64, device=dev())
    st = torch.tensor([100000, 3], dtype=torch.int32, device=dev())
    x, g = (R.rng_tensor(rng, (2, 5, 3, 80), "f32")[0].to(dev()) for _ in "xg")
    for layout in ("half", "interleaved"):
        y = fgq.fgq_rope(x, tab, st, layout=layout)
        back = fgq.fgq_rope(y, tab, st, layout=layout, inverse=True)
        assert (back - x).abs().max().item() <= 2.0 ** -20 * 2 * x.abs().max().item()  # two turns of 2^-21 (|a| + |b|)
        dx = fgq.fgq_rope(g, tab, st, layout=layout, inverse=True)
        a, b = (dx.double() * x.double()).sum().item(), (g.double() * y.double()).sum().item()
        assert abs(a - b) <= 2.0 ** -20 * (g.double().abs() * x.double().abs()).sum().item() * 4
        # differences: J is linear, J (x + h) - J x = J h to the roundings of three turns
        h = torch.zeros_like(x)
        h[0, 1, 2, 3] = 1.0
        d = fgq.fgq_rope(x + h, tab, st, layout=layout) - y
        assert (d - fgq.fgq_rope(h, tab, st, layout=layout)).abs().max().item() <= 3 * 2.0 ** -21 * 2 * (x.abs().max().item() + 1)


def test_empty_and_odd_strides():
    tab = fgq.rope_table(16, device=dev())
    none = torch.zeros(0, dtype=torch.int32, device=dev())
    one = torch.tensor([7], dtype=torch.int32, device=dev())
    for shape, st in (((0, 4, 2, 16), none), ((1, 0, 2, 16), one), ((1, 4, 0, 16), one)):
        assert fgq.fgq_rope(torch.zeros(shape, device=dev()), tab, st).shape == shape
    # rows that start off 16-byte boundaries
    rng = np.random.default_rng(5)
    base = torch.from_numpy(rng.standard_normal((1, 5, 2 * 16 + 3)).astype(np.float32)).to(dev())
    x = base[:, :, 1:33].unflatten(2, (2, 16))
    y = fgq.fgq_rope(x, tab, one)
    assert torch.equal(y, fgq.fgq_rope(x.contiguous(), tab, one))
    # another stream, and a captured graph replayed on other positions
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z = fgq.fgq_rope(x, tab, one)
    side.synchronize()
    assert torch.equal(y, z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = fgq.fgq_rope(x, tab, one)
    one.fill_(1234567)
    graph.replay()
    assert torch.equal(z, fgq.fgq_rope(x, tab, one))


def test_refusals():
    x = torch.zeros((1, 2, 3, 8), device=dev())
    tab = fgq.rope_table(8, device=dev())
    st = torch.zeros(1, dtype=torch.int32, device=dev())
    with pytest.raises(ValueError):
        fgq.fgq_rope(x, tab, st, layout="pairs")
    with pytest.raises(ValueError):
        fgq.fgq_rope(x.transpose(2, 3), tab, st)
    with pytest.raises(ValueError):
        fgq.fgq_rope(x, tab, st, out=torch.zeros((1, 2, 3, 4), device=dev()))
    with pytest.raises(ValueError):
        fgq.fgq_rope(x, tab, torch.zeros(2, dtype=torch.int32, device=dev()))
    with pytest.raises(TypeError):
        fgq.fgq_rope(x, tab.to(torch.int32), st)
    with pytest.raises(fgq.FGQError):
        fgq.fgq_rope(x, fgq.rope_table(16, device=dev()), st)
    with pytest.raises(ValueError):
        fgq.rope_table(8, scaling="other")
    with pytest.raises(fgq.FGQError):
        fgq.rope_table(7)
