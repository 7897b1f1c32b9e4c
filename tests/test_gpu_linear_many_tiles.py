"""The many-token product where a pair of SMs takes several tiles (both accumulators, the hand-over between tiles), in tiles of
256 and of 128 tokens; the quantizer that gives a warp a token; with remainders in tokens and channels."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_linear_w8a8 import weights

pytestmark = pytest.mark.gpu


# 76 pairs, tiles of 256 channels.  Tiles of 256 tokens: 9 x 8 = 72, one a pair; 17 x 11 = 187, two or three a pair, in
# five and in nine K-tiles, so that the ring of six stages is in another phase at each tile; 79 x 2 = 158.  Tiles of 128
# tokens (up to 128 tokens, or at most 38 tiles of 256): 80 and 157 of them.
@pytest.mark.parametrize("P,K,M", [(2100, 200, 1800), (4100, 264, 2700), (4097, 576, 2561), (20000, 72, 300), (9000, 65, 257),
                                   (100, 264, 20300), (128, 72, 40001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product(P, K, M, dtype):
    rng = np.random.default_rng(P + K + M)
    wq, ws, wt, st = weights(rng, M, K)
    q = rng.integers(-127, 128, (P, K)).astype(np.int8)
    sx = np.exp(rng.uniform(-6, 0, P)).astype(np.float32)
    bias = rng.standard_normal(M).astype(np.float32)
    y = torch.full((P, M), float("nan"), dtype=R.TYPES[dtype], device=dev())
    args = (torch.from_numpy(q).to(dev()), torch.from_numpy(sx).to(dev()), wt, st)
    fgq.fgq_gemm_w8a8(*args, bias=torch.from_numpy(bias).to(dev()), dtype=y.dtype, y=y)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.linear(q, sx, wq, ws, bias, dtype)
    R.check(y.float().cpu().numpy(), want, bound, "product")
    # the same bits again and again
    for _ in range(3):
        assert torch.equal(y, fgq.fgq_gemm_w8a8(*args, bias=torch.from_numpy(bias).to(dev()), dtype=y.dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K", [(1300, 64), (1301, 200), (2500, 2048), (1217, 1000), (1300, 2056)])
def test_quantize_many_tokens(P, K, dtype):
    rng = np.random.default_rng(P + K)
    t, x = R.to_type(rng.standard_normal((P, K)) * np.exp(rng.uniform(-4, 4, (P, 1))), dtype, dev())
    t[P - 1], x[P - 1] = 0, 0
    q, s = fgq.fgq_quantize_tokens(t)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    wq, ws = R.quantize8(x)
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
    t[5, K - 1] = float("nan")
    q, s = fgq.fgq_quantize_tokens(t)
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_NONFINITE
    wq[5], ws[5] = 0, 0
    assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("P,K,M", [(1300, 264, 2700), (2100, 1000, 1800)])
def test_linear(P, K, M, dtype):
    rng = np.random.default_rng(P)
    wq, ws, wt, st = weights(rng, M, K)
    x, xv = R.to_type(rng.standard_normal((P, K)), dtype, dev())
    y = fgq.fgq_linear_w8a8(x, wt, st)
    q, s = fgq.fgq_quantize_tokens(x)
    assert torch.equal(y, fgq.fgq_gemm_w8a8(q, s, wt, st, dtype=x.dtype))
    want, bound = R.linear(*R.quantize8(xv), wq, ws, None, dtype)
    R.check(y.float().cpu().numpy(), want, bound, "linear")
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_wait_expiry_with_several_tiles():
    x = torch.randn((4100, 264), device=dev(), dtype=torch.bfloat16)
    w = torch.randint(-127, 128, (2700, 264), dtype=torch.int8, device=dev())
    s = torch.ones(2700, device=dev())
    want = fgq.fgq_linear_w8a8(x, w, s)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    prev = fgq.fgq_debug_set_wait_limit_us(0)
    try:
        fgq.fgq_linear_w8a8(x, w, s)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_TIMEOUT
    finally:
        fgq.fgq_debug_set_wait_limit_us(prev)
    for _ in range(3):
        assert torch.equal(fgq.fgq_linear_w8a8(x, w, s), want)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_calls_in_quick_succession():
    """Blocks of the next call, and of another kernel with as much shared memory, start where a pair has just left: nothing that
    the pair had under way may reach them."""
    g = torch.Generator(device=dev())
    g.manual_seed(4)
    calls = []
    for P, K, M in ((700, 520, 1800), (4100, 264, 2700), (130, 1024, 260)):
        x = torch.randn((P, K), generator=g, device=dev()).to(torch.bfloat16)
        w = torch.randint(-127, 128, (M, K), generator=g, device=dev(), dtype=torch.int8)
        calls.append((x, w, torch.ones(M, device=dev())))
    cache = R.Cache(np.random.default_rng(4), 1, [600], 1, 128, 64, 16)
    cache_t, table = cache.tensors(dev())
    q = torch.randn((1, 600, 4, 128), generator=g, device=dev()).to(torch.bfloat16)
    n = torch.tensor([600], dtype=torch.int32, device=dev())

    def all_of_them():
        return [fgq.fgq_linear_w8a8(*c) for c in calls] + [fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, n)]
    want = all_of_them()
    got = [all_of_them() for _ in range(50)]
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    for ys in got:
        assert all(torch.equal(a, b) for a, b in zip(ys, want))
