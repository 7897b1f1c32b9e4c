"""Linear layers on 4-bit weights: the codes, what they stand for, and the products against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu

WHICH = [0]  # kernels that calls are restricted to


@pytest.fixture
def kernels(request):
    """1: the kernels of few tokens, 2: of many, 0: by sizes and type."""
    prev = fgq.fgq_debug_set_linear_w4_kernel(request.param)
    WHICH[0] = request.param
    yield request.param
    WHICH[0] = 0
    assert fgq.fgq_debug_set_linear_w4_kernel(prev) == request.param


def many(dtype, P, K, M):
    """Whether the product for many tokens runs: its bound is the wider one."""
    if WHICH[0]:
        return WHICH[0] == 2
    few, tile, most = (8, 8, 1 << 27) if dtype == "f32" else (16, 32, 1 << 30)
    return P > few and -(-P // tile) * tile * K * M > most


@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("shape", [(1, 1), (16, 128), (17, 129), (3, 40, 200), (2, 5, 31)])
def test_quantize_and_read(G, shape):
    rng = np.random.default_rng(G)
    w = (rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[:-1] + (1,)) * 3)).astype(np.float32)
    w[..., 0, :] = 0
    w[..., -1, -1] = 1e30
    got = fgq.fgq_quantize_weights_w4(torch.from_numpy(w).to(dev()), G)
    c, s = R.quantize_w4(w, G)
    codes, sc = R.pack_w4(c, s, G)
    assert np.array_equal(got.codes.cpu().numpy(), codes)
    assert np.array_equal(got.scales.view(torch.int16).cpu().numpy().view(np.uint16), sc)
    back = fgq.fgq_read_weights_w4(got)
    assert np.array_equal(back.cpu().numpy(), R.dequantize_w4(c, s, G).astype(np.float32))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_quantize_nonfinite_and_halves():
    w = np.zeros((2, 128), np.float32)
    w[0, :64] = np.arange(64) % 15 / 2.0  # halves: to even; the largest, 7, has code 7
    w[0, 70], w[1, 3] = np.nan, -np.inf
    w[1, 64:] = 3.5
    got = fgq.fgq_quantize_weights_w4(torch.from_numpy(w).to(dev()), 64)
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_NONFINITE
    back = fgq.fgq_read_weights_w4(got).cpu().numpy()
    assert np.array_equal(back[0, :64], np.rint(w[0, :64])) and not back[0, 64:].any() and not back[1, :64].any()
    assert np.all(back[1, 64:] == 3.5)


def run(rng, P, K, M, G, dtype, bias=True, ld=0, fill=0, spread=0.3, scale=1.0):
    x, x64 = R.rng_tensor(rng, (P, K + ld), dtype, scale)
    c, s = R.random_w4(rng, (M, K), G, spread)
    w = R.weights(c, s, G, dev(), fill)
    b = rng.standard_normal(M).astype(np.float32) if bias else None
    y = fgq.fgq_linear_w4(x.to(dev())[:, :K], w, bias=None if b is None else torch.from_numpy(b).to(dev()))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.linear(x64[:, :K], R.dequantize_w4(c, s, G), G, None if b is None else b.astype(np.float64), dtype,
                           many=many(dtype, P, K, M))
    R.check(y.double().cpu().numpy(), want, bound, f"linear {P} x {K} -> {M}")
    return y


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("P,K,M", [(1, 1, 1), (1, 128, 16), (1, 4096, 64), (2, 1000, 33), (3, 136, 40), (8, 1111, 999), (9, 512, 128),
                                   (17, 257, 50), (31, 2048, 48), (33, 640, 100), (64, 384, 31), (65, 384, 300), (130, 1000, 257)])
def test_products(kernels, dtype, G, P, K, M):
    run(np.random.default_rng(P * K + M), P, K, M, G, dtype, bias=M % 2 == 0)


@pytest.mark.parametrize("kernels", [1, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G,P,K,M", [(64, 9, 4096, 1100), (32, 16, 8192, 520), (128, 40, 8200, 130), (64, 70, 2048, 2100),
                                     (32, 130, 1000, 4300), (128, 300, 1111, 3800), (64, 260, 5120, 8200), (64, 1025, 520, 8000), (64, 18, 8192, 4100)])
def test_many(kernels, dtype, G, P, K, M):
    """Tiles of 64, 128 and 256 tokens, K in one piece and in parts, the last of them short."""
    run(np.random.default_rng(P + K), P, K, M, G, dtype, bias=M % 200 == 0)


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_very_many_tokens(kernels, dtype):
    """More rows than a launch has blocks in its second dimension, of a small matrix."""
    run(np.random.default_rng(3), 70001, 72, 40, 64, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("P,K,M,ld", [(1025, 4096, 2056, 0), (1030, 2500, 3360, 3), (1100, 2048, 4112, 8)])
def test_expanded(dtype, P, K, M, ld):
    """So many tokens that the weights are expanded once: tokens in place, copied, and with rows apart."""
    run(np.random.default_rng(P), P, K, M, 32, dtype, bias=ld > 0, ld=ld, fill=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K", [(1, 16384), (4, 14336), (7, 12000), (8, 16400), (12, 6000), (16, 9000), (32, 9000)])
def test_long_rows(dtype, P, K):
    """Tokens that a block's shared memory holds only in part, or not at all."""
    for M, G in ((100, 64), (2500, 32)):
        run(np.random.default_rng(K), P, K, M, G, dtype)


@pytest.mark.parametrize("kernels", [2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,M", [(40, 4096, 260), (200, 2048, 2100), (1000, 1024, 8200)])
def test_waits_that_run_out(kernels, dtype, P, K, M):
    """A limit of a few microseconds for each wait: an error status, and the next calls are right."""
    rng = np.random.default_rng(P)
    x = R.rng_tensor(rng, (P, K), dtype)[0].to(dev())
    w = R.weights(*R.random_w4(rng, (M, K), 64), 64, dev())
    want = fgq.fgq_linear_w4(x, w)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    seen = set()
    for limit in (0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 40, 80):
        for _ in range(3):
            prev = fgq.fgq_debug_set_wait_limit_us(limit)
            try:
                y = fgq.fgq_linear_w4(x, w)
            finally:
                fgq.fgq_debug_set_wait_limit_us(prev)
            status = fgq.fgq_stream_status()
            assert status in (fgq.FGQ_OK, fgq.FGQ_ERR_TIMEOUT)
            assert status != fgq.FGQ_OK or torch.equal(y, want)
            seen.add(status)
            assert torch.equal(fgq.fgq_linear_w4(x, w), want)
            assert fgq.fgq_stream_status() == fgq.FGQ_OK
    assert fgq.FGQ_ERR_TIMEOUT in seen


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P", [1, 5, 20, 70])
def test_strides_and_padding(kernels, dtype, P):
    """Rows apart, off 16-byte boundaries; whatever codes stand past the matrix."""
    rng = np.random.default_rng(P)
    for ld in (8, 1, 5):
        run(rng, P, 200, 40, 64, dtype, ld=ld, fill=5)
    run(rng, P, 205, 40, 64, dtype, fill=-3)
    if P < 40:  # rows of a large matrix that are not in pieces of 16 bytes
        run(rng, P, 4099, 4200, 64, dtype)
    for G, K in ((32, 129), (32, 200), (64, 257), (128, 130), (32, 96)):
        run(rng, P, K, 40, G, dtype, fill=6)


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_accuracy(kernels, dtype):
    """How far from 64 bits over many values: fp32 within 1e-6 of the output's norm, 16-bit types at their output's rounding.
    (Each rounding is uniform within half a step of a value of random mantissa: 0.41 of the largest, root mean square.)"""
    rng = np.random.default_rng(7)
    for P in (4, 40, 100):
        x, x64 = R.rng_tensor(rng, (P, 2048), dtype)
        c, s = R.random_w4(rng, (512, 2048), 64)
        y = fgq.fgq_linear_w4(x.to(dev()), R.weights(c, s, 64, dev())).double().cpu().numpy()
        want = x64 @ R.dequantize_w4(c, s, 64).T
        rel = np.linalg.norm(y - want) / np.linalg.norm(want)
        assert rel <= {"f32": 1e-6, "bf16": 0.5 * 2.0 ** -8, "f16": 0.5 * 2.0 ** -11}[dtype], rel


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P", [3, 90])
def test_magnitudes(kernels, dtype, P):
    """Scales that differ by 2^20 within a row, tokens far from 1."""
    rng = np.random.default_rng(11)
    run(rng, P, 512, 40, 32, dtype, spread=4.0, bias=False)
    for scale in (1e-3, 1e3) + (() if dtype == "f16" else (1e-20, 1e20)):
        run(rng, P, 512, 40, 32, dtype, scale=scale, bias=False)


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P", [6, 80])
def test_nonfinite_tokens(kernels, dtype, P):
    rng = np.random.default_rng(5)
    x = R.rng_tensor(rng, (P, 300), dtype)[0].to(dev())
    c, s = R.random_w4(rng, (70, 300), 64)
    w = R.weights(c, s, 64, dev())
    y0 = fgq.fgq_linear_w4(x, w)
    x[1, 200], x[4, 0] = float("nan"), -float("inf")
    y1 = fgq.fgq_linear_w4(x, w)
    keep = [p for p in range(P) if p not in (1, 4)]
    assert torch.equal(y0[keep], y1[keep])
    assert not torch.isfinite(y1[[1, 4]]).any()
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


@pytest.mark.parametrize("kernels", [0, 2], indirect=True)
def test_in_place_empty_streams_graphs(kernels):
    rng = np.random.default_rng(6)
    c, s = R.random_w4(rng, (256, 256), 64)
    w = R.weights(c, s, 64, dev())
    for dtype in ("f32", "bf16"):
        for P in (1, 12, 100):
            x = R.rng_tensor(rng, (P, 256), dtype)[0].to(dev())
            y = fgq.fgq_linear_w4(x, w)
            z = x.clone()
            assert torch.equal(fgq.fgq_linear_w4(z, w, y=z), y)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                z = fgq.fgq_linear_w4(x, w)
            side.synchronize()
            assert torch.equal(z, y)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                z = fgq.fgq_linear_w4(x, w)
            x.neg_()
            graph.replay()
            assert torch.equal(z, fgq.fgq_linear_w4(x, w)) and torch.equal(z, -y)
    assert fgq.fgq_linear_w4(x[:0], w).shape == (0, 256)
    c, s = np.zeros((20, 0), np.int8), np.zeros((20, 0), np.float32)
    none = fgq.W4Weights(torch.zeros((2, 0, 1024), dtype=torch.uint8, device=dev()),
                         torch.zeros((2, 0, 16, 2), dtype=torch.bfloat16, device=dev()), 20, 0)
    b = torch.arange(20, dtype=torch.float32, device=dev())
    assert torch.equal(fgq.fgq_linear_w4(torch.zeros((3, 0), device=dev()), none, bias=b), b.expand(3, 20))
    assert not fgq.fgq_linear_w4(torch.zeros((3, 0), device=dev()), none).any()


def test_no_scratch():
    """Calls that need a temporary say so where there is none, and those that do not run."""
    rng = np.random.default_rng(8)
    c, s = R.random_w4(rng, (64, 256), 64)
    w = R.weights(c, s, 64, dev())
    prev = fgq.fgq_debug_set_scratch_limit(0)
    try:
        for dtype in ("bf16", "f32"):
            fgq.fgq_linear_w4(R.rng_tensor(rng, (4, 256), dtype)[0].to(dev()), w)
        buf = torch.zeros((4, 256), device=dev())
        many = R.rng_tensor(rng, (100, 256), "bf16")[0].to(dev())
        for x, y, which in ((many, None, 2), (buf, buf.view(-1)[:256].view(4, 64), 0)):
            fgq.fgq_debug_set_linear_w4_kernel(which)
            with pytest.raises(fgq.FGQError) as e:
                fgq.fgq_linear_w4(x, w, y=y)
            assert e.value.code == fgq.FGQ_ERR_CUDA
    finally:
        fgq.fgq_debug_set_linear_w4_kernel(0)
        fgq.fgq_debug_set_scratch_limit(prev)


def test_kernel_setting():
    for which in (-1, 3):
        assert fgq.fgq_debug_set_linear_w4_kernel(which) == -1
    assert fgq.fgq_debug_set_linear_w4_kernel(1) == 0 and fgq.fgq_debug_set_linear_w4_kernel(0) == 1


def test_refusals():
    w = fgq.fgq_quantize_weights_w4(torch.zeros((20, 150), device=dev()))
    x = torch.zeros((2, 150), device=dev())
    with pytest.raises(ValueError):
        fgq.fgq_linear_w4(x[:, :149], w)
    with pytest.raises(ValueError):
        fgq.fgq_linear_w4(x, w, bias=torch.zeros(19, device=dev()))
    with pytest.raises(ValueError):
        fgq.W4Weights(w.codes, w.scales, 33, 150)
    with pytest.raises(ValueError):
        fgq.W4Weights(w.codes, w.scales[:, :, :8], 20, 150)
    with pytest.raises(ValueError):
        fgq.fgq_quantize_weights_w4(torch.zeros((20, 150), device=dev()), group=16)
    with pytest.raises(fgq.FGQError):
        fgq.fgq_linear_w4(x, fgq.fgq_quantize_weights_w4(torch.zeros((2, 20, 150), device=dev())))
