"""Attention over the 4-bit cache against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def run(rng, B, T, Hq, Hkv, D, G, page, dtype, seq_lens, q_lens=None, causal=True, window=0, scale=None, max_len=0,
        garbage=True, scale_v=1.0, q_scale=1.5, fp16_rows=False):
    cache = R.Cache(rng, B, seq_lens, Hkv, D, G, page, garbage=garbage, scale_v=scale_v)
    (kc, kp, vc, vp), table = cache.tensors(dev())
    qt, qx = R.to_type(rng.standard_normal((B, T, Hq, D)) * q_scale, dtype, dev())
    n = torch.tensor(list(seq_lens), dtype=torch.int32, device=dev())
    nq = None if q_lens is None else torch.tensor(list(q_lens), dtype=torch.int32, device=dev())
    out = torch.full_like(qt, float("nan"))
    fgq.fgq_kv_attention(qt, fgq.KVCache(kc, kp, vc, vp), table, n, q_lens=nq, causal=causal, window=window,
                         scale=scale, max_len=max_len, out=out)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, seq_lens, q_lens, causal, window, D ** -0.5 if scale is None else scale, dtype,
                              fp16_rows)
    R.check(out.float().cpu().numpy(), want, bound, "attention")
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
def test_one_token(dtype, D, G):
    rng = np.random.default_rng(D * 7 + G)
    run(rng, 4, 1, 8, 2, D, G, 16, dtype, [1, 33, 300, 0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Hq,Hkv,T", [(1, 1, 1), (5, 5, 2), (12, 2, 3), (16, 1, 1), (24, 3, 5)])
def test_head_layouts_and_several_queries(dtype, Hq, Hkv, T):
    rng = np.random.default_rng(Hq * 100 + T)
    run(rng, 2, T, Hq, Hkv, 128, 64, 48, dtype, [70, 2])


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700, 2049])
def test_lengths(n):
    run(np.random.default_rng(n), 1, 1, 4, 1, 64, 64, 32, "f16", [n])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_split_over_many_chunks(D):
    """Long sequences beside short and empty ones: chunks with nothing to do are skipped by the join."""
    rng = np.random.default_rng(D)
    run(rng, 3, 2, 4, 1, D, 64, 64, "bf16", [5003, 0, 65], max_len=5003)


def test_longer_than_the_bound():
    """max_len only shapes the launch: the last chunk takes the rest."""
    run(np.random.default_rng(2), 2, 1, 2, 1, 64, 32, 16, "f16", [900, 411], max_len=200)


@pytest.mark.parametrize("window", [1, 2, 16, 17, 40, 1000])
@pytest.mark.parametrize("T", [1, 4])
def test_windows(window, T):
    rng = np.random.default_rng(window * 10 + T)
    run(rng, 3, T, 4, 2, 64, 64, 16, "f16", [333, 47, 3], window=window)


def test_window_over_dropped_pages():
    """Pages wholly before the window need not exist."""
    rng = np.random.default_rng(4)
    B, D, page, n, window = 1, 64, 16, 200, 30
    cache = R.Cache(rng, B, [n], 1, D, 64, page)
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((B, 2, 2, D)), "bf16", dev())
    first = n - 2 + 1 - window  # the first position that either query sees
    table[0, :first // page] = -1
    out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()),
                               window=window)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, [n], None, True, window, D ** -0.5, "bf16")
    R.check(out.float().cpu().numpy(), want, bound, "window")


def test_queries_that_see_nothing():
    """Fewer tokens than queries, queries that do not exist, empty sequences: zeros."""
    rng = np.random.default_rng(5)
    out = run(rng, 5, 6, 4, 2, 64, 32, 16, "f32", [3, 0, 40, 9, 6], q_lens=[6, 6, 2, 0, 9])
    assert not out[0, :3].any() and out[0, 3].any()
    assert not out[1].any() and not out[3].any()
    assert out[2, 1].any() and not out[2, 2:].any()


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_not_causal(dtype):
    run(np.random.default_rng(6), 2, 5, 4, 2, 128, 128, 32, dtype, [100, 33], causal=False)


@pytest.mark.parametrize("scale_v", [1e-12, 1e-3, 1e6, 1e20])
def test_value_magnitudes(scale_v):
    run(np.random.default_rng(8), 2, 1, 4, 2, 64, 32, 16, "f32", [150, 40], scale_v=scale_v)


@pytest.mark.parametrize("q_scale", [1e-30, 1e-3, 40.0])
def test_query_magnitudes(q_scale):
    run(np.random.default_rng(9), 2, 1, 4, 2, 64, 32, 16, "f32", [150, 40], q_scale=q_scale)


def test_rising_scores():
    """Scores that grow along the sequence move the reference tile after tile."""
    rng = np.random.default_rng(10)
    D, n = 64, 600
    cache = R.Cache(rng, 1, [n], 1, D, 64, 16)
    q = rng.standard_normal((1, 1, 2, D))
    u = q[0, 0, 0] / np.linalg.norm(q[0, 0, 0])
    k = np.zeros((cache.packed[0].shape[0], 1, 16, D))
    for p in range(n):
        k[cache.table[0, p // 16], 0, p % 16] = u * p * 0.15
    cache.k = R.quantize4(k.astype(np.float32), 64)
    cache.packed[0], cache.packed[1] = R.pack_codes(cache.k[0], True), R.pack_params(*cache.k[1:])
    cache_t, table = cache.tensors(dev())
    qt, qx = R.to_type(q, "f32", dev())
    out = fgq.fgq_kv_attention(qt, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()))
    want, bound = R.attention(cache, qx, [n], None, True, 0, D ** -0.5, "f32")
    R.check(out.cpu().numpy(), want, bound, "rising")


def test_strided_queries_another_stream_and_repeats():
    rng = np.random.default_rng(11)
    B, T, H, D, n = 2, 3, 4, 64, 90
    cache = R.Cache(rng, B, [n, n], 2, D, 32, 16)
    cache_t, table = cache.tensors(dev())
    fused = torch.from_numpy(rng.standard_normal((B, T, 2 * H, D)).astype(np.float32)).to(dev())
    q = fused[:, :, :H]
    lens = torch.tensor([n, n], dtype=torch.int32, device=dev())
    c = fgq.KVCache(*cache_t)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = fgq.fgq_kv_attention(q, c, table, lens)
    side.synchronize()
    b = fgq.fgq_kv_attention(q.contiguous(), c, table, lens)
    assert torch.equal(a, b) and torch.equal(b, fgq.fgq_kv_attention(q, c, table, lens))
    want, bound = R.attention(cache, q.double().cpu().numpy(), [n, n], None, True, 0, D ** -0.5, "f32")
    R.check(a.cpu().numpy(), want, bound, "strided")


def test_bad_pages_are_reported():
    rng = np.random.default_rng(12)
    cache = R.Cache(rng, 1, [40], 1, 64, 64, 16)
    cache_t, table = cache.tensors(dev())
    q = torch.randn((1, 1, 1, 64), device=dev())
    n = torch.tensor([40], dtype=torch.int32, device=dev())
    for bad in (-1, 10 ** 6):
        t = table.clone()
        t[0, 1] = bad
        fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), t, n)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_ARG
    # a length past the table
    fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([64], dtype=torch.int32, device=dev()))
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_ARG


def test_wait_expiry_is_reported():
    """A wait limit of zero expires every wait: an error status, and the next call is right again."""
    rng = np.random.default_rng(13)
    cache = R.Cache(rng, 1, [2000], 1, 128, 64, 16)
    cache_t, table = cache.tensors(dev())
    q = torch.randn((1, 1, 4, 128), device=dev(), dtype=torch.bfloat16)
    n = torch.tensor([2000], dtype=torch.int32, device=dev())
    want = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, n)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    prev = fgq.fgq_debug_set_wait_limit_us(0)
    try:
        fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, n)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_TIMEOUT
    finally:
        fgq.fgq_debug_set_wait_limit_us(prev)
    got = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, n)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK and torch.equal(got, want)


def test_no_scratch_is_reported():
    rng = np.random.default_rng(14)
    cache = R.Cache(rng, 1, [4000], 1, 64, 64, 16)
    cache_t, table = cache.tensors(dev())
    q = torch.randn((1, 1, 4, 64), device=dev(), dtype=torch.bfloat16)
    prev = fgq.fgq_debug_set_scratch_limit(16)
    try:
        with pytest.raises(fgq.FGQError):
            fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([4000], dtype=torch.int32, device=dev()))
    finally:
        fgq.fgq_debug_set_scratch_limit(prev)
