"""What stands between two blocks (norm, gate, scale, residual sum, norm) against its definition in 64 bits."""
import itertools

import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def one_norm(rng, K, kind, weight=True, bias=True, eps=1e-5):
    w = (1 + 0.3 * rng.standard_normal(K)).astype(np.float32) if weight else None
    b = (0.2 * rng.standard_normal(K)).astype(np.float32) if bias else None
    t = [None if v is None else torch.from_numpy(v).to(dev()) for v in (w, b)]
    d = [None if v is None else v.astype(np.float64) for v in (w, b)]
    return fgq.Norm(t[0], t[1], kind=kind, eps=eps), (d[0], d[1], kind, float(np.float32(eps)))


def run(rng, P, K, dtype, rdtype=None, kind="rms", post=False, pre=True, gate=None, per=0, scale=1.0, mean=0.0, ld=0, weight=True,
        bias=True, spread=1.0):
    """gate: rows of it; ld: elements of a row beyond K."""
    x, x64 = R.rng_tensor(rng, (P, K + ld), dtype, spread)
    x64 = x64[:, :K]
    if mean:
        x = (x.float() + mean).to(x.dtype)
        x64 = x.double().numpy()[:, :K]
    xd = x.to(dev())[:, :K]
    r = r64 = None
    if rdtype:
        r, r64 = R.rng_tensor(rng, (P, K + ld), rdtype, 3 * spread)
        r, r64 = r.to(dev())[:, :K], r64[:, :K]
    g = g64 = None
    if gate:
        g, g64 = R.rng_tensor(rng, (gate, K + ld), dtype)
        g, g64 = g.to(dev())[:, :K], g64[:, :K]
    npre, dpre = one_norm(rng, K, kind, weight, bias) if pre else (None, None)
    npost, dpost = one_norm(rng, K, kind, weight, bias) if post else (None, None)
    s, y = fgq.fgq_add_norm(xd, r, npre, post=npost, gate=g, tokens_per_gate=per, scale=scale)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want = R.add_norm(x64, r64, dpre, dpost, g64, per or max(P, 1), scale, dtype, rdtype or dtype)
    R.check(s.double().cpu().numpy(), *want[0], "residual")
    if pre:
        R.check(y.double().cpu().numpy(), *want[1], "y")
    else:
        assert y is None


@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", None)])
@pytest.mark.parametrize("K", [1, 7, 64, 96, 512, 1000, 1001, 2048, 2056, 4096, 4104, 8192, 9000, 16384])
def test_sizes(dtype, rdtype, K):
    rng = np.random.default_rng(K)
    for kind, post in itertools.product(("rms", "layer"), (False, True)):
        if K == 1 and kind == "layer":
            continue  # 0 / sqrt(eps)
        run(rng, 5, K, dtype, rdtype, kind, post, gate=2, per=3, scale=0.5)


@pytest.mark.parametrize("K", [16385, 20000, 70001])
def test_long_rows(K):
    rng = np.random.default_rng(K)
    for kind in ("rms", "layer"):
        run(rng, 2, K, "bf16", "f32", kind, post=True, gate=2, per=1, scale=0.7)


@pytest.mark.parametrize("K", [500, 1024, 2048, 4096])
def test_many_rows(K):
    """The forms for many rows."""
    rng = np.random.default_rng(K)
    run(rng, 1300, K, "bf16", "bf16", "rms", post=True, gate=1300, per=1)
    run(rng, 1301, K, "f16", "f16", "layer")


def test_parts_left_out():
    rng = np.random.default_rng(0)
    for pre, post, gate, weight, bias in itertools.product((False, True), (False, True), (None, 1), (False, True), (False, True)):
        run(rng, 3, 136, "bf16", "bf16", "rms", post, pre, gate, 0, 1.0, weight=weight, bias=bias)


def test_strides_and_places():
    """Rows apart, off 16-byte boundaries; the sum in the residual's place and y in x's."""
    rng = np.random.default_rng(1)
    for ld in (8, 3, 1):
        run(rng, 9, 256, "bf16", "f32", "layer", post=True, gate=9, per=1, ld=ld)
    for K in (512, 515, 17000):
        x = R.rng_tensor(rng, (4, K), "bf16")[0].to(dev())
        r = R.rng_tensor(rng, (4, K), "bf16")[0].to(dev())
        n, _ = one_norm(rng, K, "rms")
        s, y = fgq.fgq_add_norm(x, r, n, post=n)
        x2, r2 = x.clone(), r.clone()
        s2, y2 = fgq.fgq_add_norm(x2, r2, n, post=n, residual_out=r2, y=x2)
        assert s2 is r2 and y2 is x2 and torch.equal(s, r2) and torch.equal(y, x2)


def test_large_mean_and_magnitudes():
    """A mean of 1000 costs a layer norm none of its bits; magnitudes up to 1e17 and down to 1e-15, where eps rules."""
    rng = np.random.default_rng(2)
    run(rng, 4, 4096, "f32", "f32", "layer", mean=1000.0)
    run(rng, 4, 4096, "f32", None, "layer", mean=1000.0, post=True)
    for spread in (1e17, 1e-15):
        run(rng, 4, 300, "bf16", "f32", "rms", spread=spread)
        run(rng, 4, 300, "f32", "f32", "rms", post=True, spread=spread)


def test_nonfinite_rows():
    """A token with NaN or Inf gives NaN; its neighbours are as without it; zeros give the bias."""
    rng = np.random.default_rng(3)
    for K in (300, 512, 4096, 17000):
        x = R.rng_tensor(rng, (5, K), "f32")[0].to(dev())
        r = R.rng_tensor(rng, (5, K), "f32")[0].to(dev())
        for kind in ("rms", "layer"):
            n, (_, b, _, _) = one_norm(rng, K, kind)
            s0, y0 = fgq.fgq_add_norm(x, r, n, post=n)
            x1 = x.clone()
            x1[1, K // 2], x1[3, 0] = float("nan"), float("inf")
            s1, y1 = fgq.fgq_add_norm(x1, r, n, post=n)
            for p in (0, 2, 4):
                assert torch.equal(s0[p], s1[p]) and torch.equal(y0[p], y1[p])
            assert torch.isnan(y1[1]).all() and torch.isnan(y1[3]).all()
            _, y = fgq.fgq_add_norm(torch.zeros_like(x), torch.zeros_like(r), n)
            assert np.array_equal(y.cpu().numpy(), np.broadcast_to(b.astype(np.float32), (5, K)))


def test_streams_graphs_empty():
    rng = np.random.default_rng(4)
    x = R.rng_tensor(rng, (6, 640), "bf16")[0].to(dev())
    r = R.rng_tensor(rng, (6, 640), "bf16")[0].to(dev())
    n, _ = one_norm(rng, 640, "rms", bias=False)
    s, y = fgq.fgq_add_norm(x, r, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s1, y1 = fgq.fgq_add_norm(x, r, n)
    side.synchronize()
    assert torch.equal(s, s1) and torch.equal(y, y1)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s1, y1 = fgq.fgq_add_norm(x, r, n)
    x.mul_(-0.5)
    graph.replay()
    s, y = fgq.fgq_add_norm(x, r, n)
    assert torch.equal(s, s1) and torch.equal(y, y1)
    s, y = fgq.fgq_add_norm(x[:0], r[:0], n)
    assert s.shape == y.shape == (0, 640)


def test_refusals():
    x = torch.zeros((4, 16), device=dev())
    n = fgq.Norm(torch.ones(16, device=dev()))
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, x[:, :8], n)
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, x, fgq.Norm(torch.ones(8, device=dev())))
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, x, n, gate=torch.ones((1, 16), device=dev()), tokens_per_gate=2)
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, x, n, gate=torch.ones((4, 16), device=dev(), dtype=torch.bfloat16), tokens_per_gate=1)
    with pytest.raises(ValueError):
        fgq.fgq_add_norm(x, x, None, y=torch.empty_like(x))
    with pytest.raises(fgq.FGQError):
        fgq.fgq_add_norm(x, x.to(torch.bfloat16), n)
    with pytest.raises(ValueError):
        fgq.Norm(kind="batch")
