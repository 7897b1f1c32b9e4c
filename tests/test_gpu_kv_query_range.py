"""Queries over the whole range of their types: the largest magnitudes, and scores far below zero."""
import numpy as np
import pytest
import torch

import _decoder as R
import _kv_content as C
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def attend(cache, q, n, scale, which):
    cache_t, table = cache.tensors(dev())
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()),
                                   scale=scale)
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    return out.float().cpu().numpy()


@pytest.mark.parametrize("n", [100, 700])
@pytest.mark.parametrize("magnitude", [3e34, 1e36, 8e36])
@pytest.mark.parametrize("dtype,which", [("f32", 1), ("bf16", 1), ("bf16", 2)])
def test_large_queries(n, magnitude, dtype, which):
    """Scores of ordinary size: the scale takes the queries' magnitude back."""
    rng = np.random.default_rng(n)
    D = 64
    cache = R.Cache(rng, 1, [n], 2, D, 32, 16)
    x = rng.standard_normal((1, 2, 4, D)) * magnitude
    x[..., 3] = 3.3e38 * np.sign(x[..., 3]) * (magnitude == 8e36)
    q, qx = R.to_type(x, dtype, dev())
    scale = float(np.float32(0.1 / magnitude))
    got = attend(cache, q, n, scale, which)
    want, bound = R.attention(cache, qx, [n], None, True, 0, scale, dtype, fp16_rows=which == 2)
    R.check(got, want, bound, "large queries")


@pytest.mark.parametrize("n", [100, 700])
@pytest.mark.parametrize("score", [-1e29, -1e31, -1e36])
@pytest.mark.parametrize("dtype,which", [("f32", 1), ("bf16", 1), ("bf16", 2)])
def test_scores_far_below_zero(n, score, dtype, which):
    """The same key at every position: equal scores, whatever their size, so the output is the values' mean."""
    rng = np.random.default_rng(n)
    D = 64
    k = np.ones((n, 1, D))
    v = rng.standard_normal((n, 1, D))
    cache = C.cache_of(rng, k, v, 32)
    q, qx = R.to_type(np.full((1, 1, 1, D), score), dtype, dev())
    got = attend(cache, q, n, 1.0 / D, which)
    want, bound = R.attention(cache, np.zeros_like(qx), [n], None, True, 0, 1.0 / D, dtype, fp16_rows=which == 2)
    R.check(got, want, bound, "scores")
