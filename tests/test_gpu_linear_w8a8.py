"""Per-token 8-bit quantization, bit for bit, and the 8-bit product with token and channel scales."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def weights(rng, M, K):
    wq = rng.integers(-127, 128, (M, K)).astype(np.int8)
    ws = (2.0 ** rng.integers(-12, -3, M)).astype(np.float32)
    return wq, ws, torch.from_numpy(wq).to(dev()), torch.from_numpy(ws).to(dev())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K", [(1, 1), (3, 7), (2, 64), (5, 1000), (4, 8192), (2, 8200), (2, 20001)])
def test_quantize_tokens(dtype, P, K):
    rng = np.random.default_rng(P * K)
    t, x = R.to_type(rng.standard_normal((P, K)) * np.exp(rng.uniform(-4, 4, (P, 1))), dtype, dev())
    q, s = fgq.fgq_quantize_tokens(t)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    wq, ws = R.quantize8(x)
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)


def test_quantize_tokens_special_rows():
    x = torch.randn((6, 40), device=dev())
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 0] = -float("inf")
    x[4] = torch.linspace(-3.3e38, 3.3e38, 40, dtype=torch.float64).float()  # fp32 steps would overflow
    x[5] = torch.linspace(-1e-40, 2e-41, 40)
    q, s = fgq.fgq_quantize_tokens(x)
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_NONFINITE
    assert not q[1:4].any() and not s[1:4].any()
    for i in (0, 4, 5):
        r = x[i].double().cpu().numpy()
        amax = np.abs(r).max()
        assert np.array_equal(q[i].cpu().numpy(), np.rint(127 * r / amax).astype(np.int8))
        assert s[i].item() == np.float32(np.float32(amax) / np.float32(127))


@pytest.mark.parametrize("stride", [41, 48])
def test_quantize_tokens_strided_rows(stride):
    x = torch.randn((5, stride), device=dev())[:, :40]
    q, s = fgq.fgq_quantize_tokens(x)
    q2, s2 = fgq.fgq_quantize_tokens(x.contiguous())
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,M", [(1, 1, 1), (1, 4096, 48), (2, 100, 33), (7, 1040, 130), (8, 64, 16), (9, 333, 17),
                                   (17, 512, 40), (33, 1000, 129), (64, 64, 64), (70, 2751, 200), (130, 1024, 260),
                                   (257, 640, 136), (300, 4099, 1000), (600, 65, 700)])
def test_product(dtype, P, K, M):
    rng = np.random.default_rng(P + K + M)
    wq, ws, wt, st = weights(rng, M, K)
    q = rng.integers(-127, 128, (P, K)).astype(np.int8)
    sx = np.exp(rng.uniform(-6, 0, P)).astype(np.float32)
    bias = rng.standard_normal(M).astype(np.float32) if (P + M) % 2 else None
    y = torch.full((P, M), float("nan"), dtype=R.TYPES[dtype], device=dev())
    fgq.fgq_gemm_w8a8(torch.from_numpy(q).to(dev()), torch.from_numpy(sx).to(dev()), wt, st,
                      bias=None if bias is None else torch.from_numpy(bias).to(dev()), dtype=y.dtype, y=y)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.linear(q, sx, wq, ws, bias, dtype)
    R.check(y.float().cpu().numpy(), want, bound, "product")


@pytest.mark.parametrize("P", [1, 8, 40, 200])
def test_largest_sums(P):
    """Every product at its largest: exact up to K = 1040, then off by the accumulator's rounding alone."""
    for K in (1040, 8192):
        q = np.full((P, K), -127, np.int8)
        wq = np.full((80, K), 127, np.int8)
        one = np.ones(80, np.float32)
        y = fgq.fgq_gemm_w8a8(torch.from_numpy(q).to(dev()), torch.ones(P, device=dev()), torch.from_numpy(wq).to(dev()),
                              torch.from_numpy(one).to(dev()))
        exact = -127.0 * 127 * K
        assert np.all(np.abs(y.double().cpu().numpy() - exact) <= (0 if K == 1040 else abs(exact) * K / 16 * 2.0 ** -23))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,M", [(1, 4096, 64), (5, 77, 40), (3, 4096, 100), (8, 2048, 50), (31, 256, 100), (50, 1001, 130), (150, 768, 300)])
def test_linear_is_its_two_calls(dtype, P, K, M):
    rng = np.random.default_rng(P * 3 + K)
    wq, ws, wt, st = weights(rng, M, K)
    bias = torch.from_numpy(rng.standard_normal(M).astype(np.float32)).to(dev())
    x, xv = R.to_type(rng.standard_normal((P, K)), dtype, dev())
    y = fgq.fgq_linear_w8a8(x, wt, st, bias=bias)
    q, s = fgq.fgq_quantize_tokens(x)
    assert torch.equal(y, fgq.fgq_gemm_w8a8(q, s, wt, st, bias=bias, dtype=x.dtype))
    qn, sn = R.quantize8(xv)
    want, bound = R.linear(qn, sn, wq, ws, bias.cpu().numpy(), dtype)
    R.check(y.float().cpu().numpy(), want, bound, "linear")
    # rows of a wider tensor, on another stream
    wide = torch.zeros((P, K + 24), dtype=x.dtype, device=dev())
    wide[:, 8:8 + K] = x
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y2 = fgq.fgq_linear_w8a8(wide[:, 8:8 + K], wt, st, bias=bias, stream=side)
    side.synchronize()
    assert torch.equal(y, y2)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_weights_of_the_library():
    """Weights from fgq_quantize_weights_w8."""
    w = torch.randn((96, 200), device=dev())
    wq, ws = fgq.fgq_quantize_weights_w8(w)
    x = torch.randn((40, 200), device=dev())
    y = fgq.fgq_linear_w8a8(x, wq, ws)
    # the float product, within the two quantizations' half steps
    half = 0.5 * (x.abs().amax(1, keepdim=True) / 127) @ (w.abs().sum(1)[None]) + 0.5 * x.abs().sum(1, keepdim=True) * ws
    assert bool(((y - x @ w.t()).abs() <= 1.05 * half + 1e-4).all())


def test_empty_and_zero():
    w = torch.ones((8, 16), dtype=torch.int8, device=dev())
    s = torch.ones(8, device=dev())
    assert fgq.fgq_linear_w8a8(torch.empty((0, 16), device=dev()), w, s).shape == (0, 8)
    bias = torch.arange(8, dtype=torch.float32, device=dev())
    y = fgq.fgq_linear_w8a8(torch.zeros((3, 16), device=dev()), w, s, bias=bias)
    assert torch.equal(y, bias.expand(3, 8))
    # no features: the bias alone
    y = fgq.fgq_linear_w8a8(torch.empty((40, 0), device=dev()), torch.empty((8, 0), dtype=torch.int8, device=dev()), s,
                            bias=bias)
    assert torch.equal(y, bias.expand(40, 8))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_wait_expiry_is_reported():
    x = torch.randn((300, 512), device=dev(), dtype=torch.bfloat16)
    w = torch.randint(-127, 128, (256, 512), dtype=torch.int8, device=dev())
    s = torch.ones(256, device=dev())
    want = fgq.fgq_linear_w8a8(x, w, s)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    prev = fgq.fgq_debug_set_wait_limit_us(0)
    try:
        fgq.fgq_linear_w8a8(x, w, s)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_TIMEOUT
    finally:
        fgq.fgq_debug_set_wait_limit_us(prev)
    assert torch.equal(fgq.fgq_linear_w8a8(x, w, s), want)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_no_scratch_is_reported():
    x = torch.randn((300, 512), device=dev())
    w = torch.zeros((256, 512), dtype=torch.int8, device=dev())
    s = torch.ones(256, device=dev())
    prev = fgq.fgq_debug_set_scratch_limit(16)
    try:
        with pytest.raises(fgq.FGQError):
            fgq.fgq_linear_w8a8(x, w, s)
    finally:
        fgq.fgq_debug_set_scratch_limit(prev)
