"""Decoding steps from a captured CUDA graph: what the calls allocate and launch inside can be captured, and a replay on new inputs
gives what the calls give."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,B,T,dtype", [(700, 1, 1, "bf16"), (5000, 2, 1, "f16"), (60000, 1, 2, "f32"), (3000, 2, 60, "bf16")])
def test_step(n, B, T, dtype):
    """Layer, cache write, attention (cluster, either join, many rows), layer."""
    rng = np.random.default_rng(n)
    Hq, Hkv, D, width = 8, 2, 64, 256
    cache = R.Cache(rng, B, [n] * B, Hkv, D, 32, 16)
    cache_t, table = cache.tensors(dev())
    c = fgq.KVCache(*cache_t)
    g = torch.Generator(device=dev())
    g.manual_seed(n)
    w1 = fgq.fgq_quantize_weights_w8(torch.randn(((Hq + 2 * Hkv) * D, width), generator=g, device=dev()) / width ** 0.5)
    w2 = fgq.fgq_quantize_weights_w8(torch.randn((width, Hq * D), generator=g, device=dev()) / (Hq * D) ** 0.5)
    x = torch.randn((B * T, width), generator=g, device=dev()).to(R.TYPES[dtype])
    ends = torch.full((B,), n, dtype=torch.int32, device=dev())
    starts = ends - T

    def step():
        q, k, v = fgq.fgq_linear_w8a8(x, *w1).view(B, T, -1, D).split([Hq, Hkv, Hkv], dim=2)
        fgq.fgq_kv_append(c, k, v, table, starts)
        o = fgq.fgq_kv_attention(q, c, table, ends, max_len=n)
        return fgq.fgq_linear_w8a8(o.view(B * T, -1), *w2)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for seed in range(3):
        g.manual_seed(seed)
        x.copy_(torch.randn(x.shape, generator=g, device=dev()))
        starts.fill_(n - T - seed)
        ends.fill_(n - seed)
        graph.replay()
        got = y.clone()
        want = step()
        assert fgq.fgq_stream_status() == fgq.FGQ_OK
        assert torch.equal(got, want)


def test_repeats_are_the_same_bits():
    """No sum's order depends on which block comes first."""
    rng = np.random.default_rng(1)
    cache = R.Cache(rng, 3, [9000, 500, 4000], 4, 128, 64, 64)
    cache_t, table = cache.tensors(dev())
    c = fgq.KVCache(*cache_t)
    n = torch.tensor([9000, 500, 4000], dtype=torch.int32, device=dev())
    for dtype in ("f32", "bf16", "f16"):
        for T in (1, 2, 70):
            q = torch.from_numpy(rng.standard_normal((3, T, 16, 128)).astype(np.float32)).to(R.TYPES[dtype]).to(dev())
            first = fgq.fgq_kv_attention(q, c, table, n)
            for _ in range(20):
                assert torch.equal(first, fgq.fgq_kv_attention(q, c, table, n))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
