"""Routing, experts' layers and the two together against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def layer(rng, E, K, F, G, Gd=None, fill=0):
    """((device weights), (64-bit weights)) of gate, up, down."""
    on, d = [], []
    for M, N, g in ((F, K, G), (F, K, G), (K, F, Gd or G)):
        c, s = R.random_w4(rng, (E, M, N), g)
        on.append(R.weights(c, s, g, dev(), fill))
        d.append(R.dequantize_w4(c, s, g))
    return on, d


@pytest.mark.parametrize("score,renormalize", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("P,K,E,top", [(1, 64, 8, 1), (5, 1000, 64, 8), (130, 300, 12, 3), (3, 37, 200, 32), (2, 512, 1024, 5), (1, 8, 1, 1)])
def test_route(score, renormalize, dtype, rdtype, P, K, E, top):
    rng = np.random.default_rng(P + E)
    x, x64 = R.rng_tensor(rng, (P, K), dtype)
    r, r64 = R.rng_tensor(rng, (E, K), rdtype, K ** -0.5)
    ids, w = fgq.fgq_route_tokens(x.to(dev()), r.to(dev()), top, score, renormalize, 1.5)
    want, g, e = R.route(x64, r64, top, score, renormalize, 1.5)
    assert np.array_equal(ids.cpu().numpy(), want)
    R.check(w.double().cpu().numpy(), g, e * g, "weights")
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_route_ties_and_nan():
    x = torch.ones((3, 16), device=dev())
    r = torch.zeros((40, 16), device=dev())
    r[[7, 20, 33]] = 1.0
    ids, w = fgq.fgq_route_tokens(x, r, 5)
    assert ids.tolist() == [[7, 20, 33, 0, 1]] * 3
    x[1, 3] = float("nan")
    ids, w = fgq.fgq_route_tokens(x, r, 5)
    assert torch.isnan(w[1]).all() and torch.isfinite(w[[0, 2]]).all() and ids[1].tolist() == [0, 1, 2, 3, 4]
    # sums that fp32 would lose: 2^24 + 1 against 2^24, in the middle of a row
    x = torch.ones((1, 64), device=dev())
    r = torch.zeros((3, 64), device=dev())
    r[:, 0], r[2, 20], r[0, 40] = 2.0 ** 24, 1.0, 2.0 ** -20
    assert fgq.fgq_route_tokens(x, r, 3)[0].tolist() == [[2, 0, 1]]


def run_experts(rng, P, K, F, E, top, G, dtype, Gd=None, ids=None, fill=0, ld=0):
    on, d = layer(rng, E, K, F, G, Gd, fill)
    x, x64 = R.rng_tensor(rng, (P, K + ld), dtype)
    if ids is None:
        ids = np.stack([rng.permutation(max(E, top))[:top] % E for _ in range(P)]).astype(np.int32)
    g = rng.random((P, ids.shape[1])).astype(np.float32)
    y = fgq.fgq_experts_w4(x.to(dev())[:, :K], torch.from_numpy(ids).to(dev()), torch.from_numpy(g).to(dev()), *on)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.experts(x64[:, :K], ids, g.astype(np.float64), np.zeros((P, 1)), *d, G, Gd or G, dtype)
    R.check(y.double().cpu().numpy(), want, bound, f"experts {P} x {K}, {F}, {E}")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,F,E,top,G", [(1, 128, 64, 4, 2, 64), (1, 1, 1, 1, 1, 32), (1, 1000, 700, 6, 3, 32), (3, 136, 40, 9, 4, 128),
                                           (8, 256, 96, 2, 1, 64), (20, 264, 33, 5, 2, 32), (40, 130, 70, 3, 3, 64),
                                           (64, 128, 128, 16, 4, 64), (129, 64, 48, 4, 2, 64), (300, 40, 24, 2, 1, 32), (2, 2048, 16, 3, 2, 64),
                                           # units cut short of 64 and 128 tokens, two passes, long rows, layers that hold few tokens or none
                                           (130, 520, 300, 3, 2, 64), (600, 130, 140, 6, 3, 128), (700, 64, 40, 5, 8, 32), (40, 4100, 36, 2, 1, 64),
                                           (24, 136, 72, 4, 2, 32), (50, 264, 130, 4, 2, 64), (200, 700, 1100, 16, 2, 64),
                                           (300, 130, 136, 2, 1, 64),
                                           (9, 64, 15000, 3, 1, 64), (6, 20000, 17, 3, 1, 128), (2, 16, 120000, 2, 1, 64)])
def test_experts(dtype, P, K, F, E, top, G):
    run_experts(np.random.default_rng(P + K), P, K, F, E, top, G, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_many_odd_calls(dtype):
    """Many choices of which some are no expert, some tokens have none or one expert often, and all are at one expert; any codes past
    the matrices; rows apart; none at all."""
    rng = np.random.default_rng(21)
    ids = rng.integers(-1, 6, (130, 3)).astype(np.int32)
    ids[5] = -1
    ids[60:70] = 3
    run_experts(rng, 130, 200, 72, 6, 3, 64, dtype, ids=ids, Gd=32, fill=4, ld=1)
    run_experts(rng, 90, 270, 140, 2, 1, 32, dtype, fill=-5)
    run_experts(rng, 150, 136, 40, 4, 1, 128, dtype, ids=np.full((150, 1), 3, np.int32), ld=8)
    run_experts(rng, 40, 128, 32, 2, 2, 32, dtype, ids=np.full((40, 2), -1, np.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_many_nonfinite_and_graphs(dtype):
    """A token with NaN leaves the others as they are; a captured call follows its inputs; two streams at once; waits that run out."""
    rng = np.random.default_rng(22)
    on, _ = layer(rng, 4, 256, 192, 64)
    x = R.rng_tensor(rng, (90, 256), dtype)[0].to(dev())
    r = R.rng_tensor(rng, (4, 256), dtype, 1 / 16)[0].to(dev())
    ids, g = fgq.fgq_route_tokens(x, r, 2)
    y = fgq.fgq_experts_w4(x, ids, g, *on)
    z = x.clone()
    z[7, 100] = float("nan")
    out = fgq.fgq_experts_w4(z, ids, g, *on)
    keep = [p for p in range(90) if p != 7]
    assert torch.equal(out[keep], y[keep]) and not torch.isfinite(out[7]).any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fgq.fgq_moe_w4(x, r, 2, *on)
    x.copy_(x.flip(0))
    graph.replay()
    assert torch.equal(out, y.flip(0))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            outs.append([fgq.fgq_moe_w4(x, r, 2, *on) for _ in range(5)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, out) for o in sum(outs, []))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    seen = set()
    for limit in (0, 1, 2, 4, 8, 16, 40):
        for _ in range(3):
            prev = fgq.fgq_debug_set_wait_limit_us(limit)
            try:
                o = fgq.fgq_moe_w4(x, r, 2, *on)
            finally:
                fgq.fgq_debug_set_wait_limit_us(prev)
            status = fgq.fgq_stream_status()
            assert status in (fgq.FGQ_OK, fgq.FGQ_ERR_TIMEOUT)
            assert status != fgq.FGQ_OK or torch.equal(o, out)
            seen.add(status)
            assert torch.equal(fgq.fgq_moe_w4(x, r, 2, *on), out)
            assert fgq.fgq_stream_status() == fgq.FGQ_OK
    assert fgq.FGQ_ERR_TIMEOUT in seen


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_experts_odd_calls(dtype):
    rng = np.random.default_rng(9)
    # choices that are no expert, tokens without any, one expert twice or three times for a token, all tokens at one expert
    ids = np.array([[0, -1, 5], [-1, -1, -1], [2, 2, 1], [7, 100, -5], [4, 4, 4], [2 ** 31 - 1, 0, -2 ** 31]], np.int32)
    run_experts(rng, 6, 200, 72, 6, 3, 64, dtype, ids=ids)
    run_experts(rng, 50, 128, 32, 4, 1, 32, dtype, ids=np.full((50, 1), 3, np.int32))
    run_experts(rng, 7, 128, 32, 4, 2, 32, dtype, ids=np.full((7, 2), 1, np.int32))
    run_experts(rng, 2, 128, 32, 4, 2, 32, dtype, ids=np.full((2, 2), -1, np.int32))
    # groups of another size in down; any codes past the matrices; strides
    run_experts(rng, 5, 200, 70, 4, 2, 32, dtype, Gd=128, fill=4)
    for ld in (8, 1):
        run_experts(rng, 5, 200, 70, 4, 2, 128, dtype, Gd=32, ld=ld)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,F,E,top,G,score,renormalize", [(1, 512, 128, 64, 8, 64, "softmax", True), (7, 136, 100, 10, 2, 32, "sigmoid", False),
                                                             (33, 256, 64, 300, 4, 128, "softmax", False), (130, 200, 40, 6, 2, 64, "sigmoid", True),
                                                             (2, 96, 33, 600, 1, 64, "softmax", True), (1, 40, 20, 1, 1, 32, "softmax", True)])
def test_layer(dtype, P, K, F, E, top, G, score, renormalize):
    rng = np.random.default_rng(P + E)
    on, d = layer(rng, E, K, F, G)
    x, x64 = R.rng_tensor(rng, (P, K), dtype)
    r, r64 = R.rng_tensor(rng, (E, K), dtype, K ** -0.5)
    y = fgq.fgq_moe_w4(x.to(dev()), r.to(dev()), top, *on, score=score, renormalize=renormalize, scale=2.5)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    ids, g, e = R.route(x64, r64, top, score, renormalize, 2.5)
    want, bound = R.experts(x64, ids, g, e, *d, G, G, dtype)
    R.check(y.double().cpu().numpy(), want, bound, "layer")
    # the same as the two calls, bit for bit
    i2, g2 = fgq.fgq_route_tokens(x.to(dev()), r.to(dev()), top, score, renormalize, 2.5)
    assert torch.equal(y, fgq.fgq_experts_w4(x.to(dev()), i2, g2, *on))


def test_nonfinite_tokens():
    """A token that holds NaN gives NaN; the others, in the same products, are as without it."""
    rng = np.random.default_rng(3)
    on, _ = layer(rng, 4, 200, 64, 64)
    for dtype in ("f32", "bf16", "f16"):
        x = R.rng_tensor(rng, (9, 200), dtype)[0].to(dev())
        r = R.rng_tensor(rng, (4, 200), dtype, 0.1)[0].to(dev())
        ids, g = fgq.fgq_route_tokens(x, r, 2)
        y0 = fgq.fgq_experts_w4(x, ids, g, *on)
        x1 = x.clone()
        x1[4, 7] = float("nan")
        y1 = fgq.fgq_experts_w4(x1, ids, g, *on)
        keep = [p for p in range(9) if p != 4]
        assert torch.equal(y0[keep], y1[keep]) and torch.isnan(y1[4]).all()
        y2 = fgq.fgq_moe_w4(x1, r, 2, *on)
        assert torch.isnan(y2[4]).all() and torch.isfinite(y2[keep]).all()
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_streams_graphs_places():
    """Another stream, a captured graph on new tokens with others' calls between replays, y in x's place, repeats bit for bit."""
    rng = np.random.default_rng(4)
    on, _ = layer(rng, 16, 256, 128, 64)
    for P, dtype in ((1, "bf16"), (9, "f16"), (70, "bf16"), (4, "f32"), (131, "bf16")):
        x = R.rng_tensor(rng, (P, 256), dtype)[0].to(dev())
        r = R.rng_tensor(rng, (16, 256), dtype, 0.1)[0].to(dev())
        call = lambda v: fgq.fgq_moe_w4(v, r, 3, *on)  # noqa: E731
        y = call(x)
        for _ in range(10):
            assert torch.equal(call(x), y)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            z = call(x)
        side.synchronize()
        assert torch.equal(z, y)
        graphs, outs, ins = [], [], []
        for k in range(2):
            xi = x.clone()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                outs.append(call(xi))
            graphs.append(graph)
            ins.append(xi)
        for k in (0, 1, 0):
            ins[k].copy_(x * (k + 2))
            graphs[k].replay()
            call(x)
            assert torch.equal(outs[k], call(x * (k + 2)))
        z = x.clone()
        assert torch.equal(fgq.fgq_moe_w4(z, r, 3, *on, y=z), y)
    # two streams at once
    streams = [torch.cuda.Stream() for _ in range(2)]
    xs = [R.rng_tensor(rng, (20, 256), "bf16")[0].to(dev()) for _ in streams]
    r = R.rng_tensor(rng, (16, 256), "bf16", 0.1)[0].to(dev())
    want = [fgq.fgq_moe_w4(v, r, 3, *on) for v in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(fgq.fgq_moe_w4(xs[k], r, 3, *on))
    torch.cuda.synchronize()
    assert all(torch.equal(v, want[k]) for k in range(2) for v in got[k])


def test_no_scratch_and_empty():
    rng = np.random.default_rng(5)
    on, _ = layer(rng, 4, 64, 32, 64)
    x = R.rng_tensor(rng, (3, 64), "bf16")[0].to(dev())
    r = R.rng_tensor(rng, (4, 64), "bf16")[0].to(dev())
    assert fgq.fgq_moe_w4(x[:0], r, 2, *on).shape == (0, 64)
    assert fgq.fgq_route_tokens(x[:0], r, 2)[0].shape == (0, 2)
    prev = fgq.fgq_debug_set_scratch_limit(0)
    try:
        with pytest.raises(fgq.FGQError) as e:
            fgq.fgq_moe_w4(x, r, 2, *on)
        assert e.value.code == fgq.FGQ_ERR_CUDA
        fgq.fgq_route_tokens(x, r, 2)  # needs none
    finally:
        fgq.fgq_debug_set_scratch_limit(prev)


def test_refusals():
    rng = np.random.default_rng(6)
    on, _ = layer(rng, 4, 64, 32, 64)
    x = torch.zeros((3, 64), device=dev())
    ids, g = torch.zeros((3, 2), dtype=torch.int32, device=dev()), torch.ones((3, 2), device=dev())
    with pytest.raises(ValueError):
        fgq.fgq_experts_w4(x, ids[:2], g[:2], *on)
    with pytest.raises(ValueError):
        fgq.fgq_experts_w4(x, ids, g[:, :1], *on)
    with pytest.raises(TypeError):
        fgq.fgq_experts_w4(x, ids.long(), g, *on)
    with pytest.raises(fgq.FGQError):
        fgq.fgq_experts_w4(x, ids, g, on[0], on[1], on[0])
    with pytest.raises(ValueError):
        fgq.fgq_moe_w4(x, torch.zeros((5, 64), device=dev()), 2, *on)
    with pytest.raises(TypeError):
        fgq.fgq_moe_w4(x, torch.zeros((4, 64), device=dev(), dtype=torch.bfloat16), 2, *on)
    with pytest.raises(ValueError):
        fgq.fgq_route_tokens(x, torch.zeros((4, 64), device=dev()), 2, score="max")
