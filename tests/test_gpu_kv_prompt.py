"""Attention of long runs of queries over the 4-bit cache (the tensor-core kernel), against the definition in
64 bits."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
@pytest.mark.parametrize("T", [40, 150])
def test_prompt(dtype, D, G, T):
    """One tile of rows and two, whole prompts and prompts over earlier tokens, every group size."""
    rng = np.random.default_rng(D + G + T)
    run(rng, 2, T, 4, 2, D, G, 16, dtype, [T, T + 77], fp16_rows=True)


@pytest.mark.parametrize("Hq,Hkv,T", [(3, 3, 70), (7, 1, 19), (16, 2, 33), (1, 1, 129)])
def test_head_layouts(Hq, Hkv, T):
    run(np.random.default_rng(T), 2, T, Hq, Hkv, 128, 64, 48, "bf16", [T + 100, T], fp16_rows=True)


@pytest.mark.parametrize("n", [64, 65, 127, 128, 129, 191, 640])
def test_lengths(n):
    run(np.random.default_rng(n), 1, 64, 2, 1, 64, 64, 32, "f16", [n], fp16_rows=True)


@pytest.mark.parametrize("window", [1, 16, 63, 64, 100, 5000])
def test_windows(window):
    run(np.random.default_rng(window), 2, 90, 2, 1, 128, 128, 16, "f16", [333, 95], window=window, fp16_rows=True)


def test_rows_that_see_nothing():
    rng = np.random.default_rng(3)
    out = run(rng, 5, 60, 2, 2, 64, 32, 16, "bf16", [30, 0, 300, 9, 60], q_lens=[60, 60, 7, 0, 99], fp16_rows=True)
    assert not out[0, :30].any() and out[0, 30].any()
    assert not out[1].any() and not out[3].any()
    assert out[2, 6].any() and not out[2, 7:].any()


def test_split_over_chunks():
    """Few tiles of rows over long sequences: the join skips chunks with nothing to do."""
    run(np.random.default_rng(4), 2, 40, 1, 1, 64, 64, 64, "bf16", [3000, 41], fp16_rows=True)
    run(np.random.default_rng(5), 1, 48, 1, 1, 256, 64, 16, "f16", [2500], window=700, fp16_rows=True)


def test_not_causal():
    run(np.random.default_rng(6), 2, 50, 2, 1, 128, 32, 32, "f16", [100, 33], causal=False, fp16_rows=True)


@pytest.mark.parametrize("scale_v", [1e-12, 1e-3, 1e6, 1e20])
def test_value_magnitudes(scale_v):
    run(np.random.default_rng(8), 1, 48, 2, 1, 64, 32, 16, "bf16", [150], scale_v=scale_v, fp16_rows=True)


def test_magnitudes_that_change_along_the_cache():
    """Values, and keys, of another magnitude in every tile, and a tile of zeros."""
    rng = np.random.default_rng(9)
    D, n, T = 64, 400, 64
    cache = R.Cache(rng, 1, [n], 1, D, 64, 16)
    kscale, vscale = np.ones(cache.k[0].shape[0]), np.ones(cache.k[0].shape[0])
    for i, p in enumerate(cache.table[0]):
        kscale[p] = [1.0, 0.03, 2.0, 1e-4][i // 4 % 4]
        vscale[p] = [1.0, 1e-3, 0.0, 30.0][i // 4 % 4]
    for which, sc in (("k", kscale), ("v", vscale)):
        x = (rng.standard_normal(cache.k[0].shape) * sc[:, None, None, None]).astype(np.float32)
        setattr(cache, which, R.quantize4(x, 64))
    cache.packed = [R.pack_codes(cache.k[0], True), R.pack_params(*cache.k[1:]), R.pack_codes(cache.v[0], False),
                    R.pack_params(*cache.v[1:])]
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((1, T, 1, D)), "f16", dev())
    out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, [n], None, True, 0, D ** -0.5, "f16", fp16_rows=True)
    R.check(out.float().cpu().numpy(), want, bound, "magnitudes")


def test_rising_scores():
    """Scores that grow along the sequence move the reference, and the sums with it, tile after tile."""
    rng = np.random.default_rng(10)
    D, n, T = 64, 600, 40
    cache = R.Cache(rng, 1, [n], 1, D, 64, 16)
    u = rng.standard_normal(D)
    u /= np.linalg.norm(u)
    k = np.zeros((cache.packed[0].shape[0], 1, 16, D))
    for p in range(n):
        k[cache.table[0, p // 16], 0, p % 16] = u * p * 0.15
    cache.k = R.quantize4(k.astype(np.float32), 64)
    cache.packed[0], cache.packed[1] = R.pack_codes(cache.k[0], True), R.pack_params(*cache.k[1:])
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(np.broadcast_to(u, (1, T, 1, D)) * 6.0, "f16", dev())
    out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()))
    want, bound = R.attention(cache, qx, [n], None, True, 0, D ** -0.5, "f16", fp16_rows=True)
    R.check(out.float().cpu().numpy(), want, bound, "rising")


def test_repeats_streams_and_strides():
    rng = np.random.default_rng(11)
    B, T, H, D, n = 2, 70, 2, 128, 200
    cache = R.Cache(rng, B, [n, n], 1, D, 64, 16)
    cache_t, table = cache.tensors(dev())
    fused = torch.from_numpy(rng.standard_normal((B, T, 2 * H, D)).astype(np.float32)).to(torch.bfloat16).to(dev())
    q, c = fused[:, :, :H], fgq.KVCache(*cache_t)
    lens = torch.tensor([n, n], dtype=torch.int32, device=dev())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = fgq.fgq_kv_attention(q, c, table, lens, stream=side)
    side.synchronize()
    b = fgq.fgq_kv_attention(q.contiguous(), c, table, lens)
    assert torch.equal(a, b) and torch.equal(b, fgq.fgq_kv_attention(q, c, table, lens))


def test_bad_pages_and_wait_expiry():
    rng = np.random.default_rng(12)
    cache = R.Cache(rng, 1, [300], 1, 64, 64, 16)
    cache_t, table = cache.tensors(dev())
    q = torch.randn((1, 64, 1, 64), device=dev()).to(torch.bfloat16)
    n = torch.tensor([300], dtype=torch.int32, device=dev())
    c = fgq.KVCache(*cache_t)
    want = fgq.fgq_kv_attention(q, c, table, n)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    bad = table.clone()
    bad[0, 3] = -1
    fgq.fgq_kv_attention(q, c, bad, n)
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_ARG
    prev = fgq.fgq_debug_set_wait_limit_us(0)
    try:
        fgq.fgq_kv_attention(q, c, table, n)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_TIMEOUT
    finally:
        fgq.fgq_debug_set_wait_limit_us(prev)
    assert torch.equal(fgq.fgq_kv_attention(q, c, table, n), want)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
