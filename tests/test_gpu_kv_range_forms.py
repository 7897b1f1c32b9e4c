"""Magnitudes of queries, scores and values, and queries that are no numbers, on every form of the two attention kernels: head sizes,
one and two tiles of rows, one chunk, clusters and both joins."""
import numpy as np
import pytest
import torch

import _decoder as R
import _kv_content as C
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu

# head_dim, group, queries, query heads, kernel
FORMS = [(64, 32, 4, 4, 1), (128, 64, 1, 8, 1), (128, 32, 4, 4, 1), (128, 128, 2, 7, 1), (256, 64, 2, 4, 1),
         (64, 64, 150, 1, 2), (128, 64, 20, 2, 2), (128, 32, 75, 2, 2), (256, 64, 20, 2, 2), (256, 128, 130, 1, 2)]


def run(rng, k, v, q, G, which, dtype, scale, max_len=0, qdef=None):
    n, _, D = k.shape
    cache = C.cache_of(rng, k, v, G)
    cache_t, table = cache.tensors(dev())
    qt, qx = R.to_type(q, dtype, dev())
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        out = fgq.fgq_kv_attention(qt, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()),
                                   scale=scale, max_len=max_len)
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx if qdef is None else qdef, [n], None, True, 0, scale, dtype, fp16_rows=which == 2)
    return out.float().cpu().numpy(), want, bound


def dtypes(which):
    return ["bf16", "f16"] if which == 2 else ["f32", "bf16", "f16"]


CASES = [f + (t,) for f in FORMS for t in dtypes(f[4])]


@pytest.mark.parametrize("D,G,T,H,which,dtype", CASES)
@pytest.mark.parametrize("n", [160, 900, 3000])
def test_large_queries(D, G, T, H, which, dtype, n):
    rng = np.random.default_rng(D + n)
    size = 6e4 if dtype == "f16" else 3e38
    q = rng.uniform(-1, 1, (1, T, H, D)) * size
    k, v = rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D))
    got, want, bound = run(rng, k, v, q, G, which, dtype, float(np.float32(4 / size / D ** 0.5)))
    R.check(got, want, bound, "large queries")


@pytest.mark.parametrize("D,G,T,H,which,dtype", [c for c in CASES if c[5] != "f16"])
@pytest.mark.parametrize("score", [-1e36, 1e10, 1e37])
@pytest.mark.parametrize("n", [160, 900, 3000])
def test_equal_scores(D, G, T, H, which, dtype, score, n):
    """The same key everywhere; values of another magnitude in every third 16 tokens."""
    rng = np.random.default_rng(D + n)
    v = rng.standard_normal((n, 1, D)) * np.where(np.arange(n) // 16 % 3 == 0, 1e3, 1.0)[:, None, None]
    q = np.full((1, T, H, D), score)
    got, want, bound = run(rng, np.ones((n, 1, D)), v, q, G, which, dtype, 1.0 / D, qdef=np.zeros_like(q))
    R.check(got, want, bound, "equal scores")


@pytest.mark.parametrize("D,G,T,H,which,dtype", [c for c in CASES if c[5] != "f16"])
@pytest.mark.parametrize("kind", ["zeros first", "zeros last", "equal", "far apart"])
@pytest.mark.parametrize("n", [160, 900])
def test_values(D, G, T, H, which, dtype, kind, n):
    rng = np.random.default_rng(D + n)
    t = np.arange(n)
    size = {"zeros first": np.where(t < n // 2, 0, 1e28), "zeros last": np.where(t > n // 3, 0, 1e28),
            "equal": np.full(n, 2.0 ** 90), "far apart": np.where(t % 5 == 0, 1e22, 1e-2)}[kind][:, None, None]
    v = size * (np.ones((n, 1, D)) if kind == "equal" else rng.standard_normal((n, 1, D)))
    got, want, bound = run(rng, rng.standard_normal((n, 1, D)), v, rng.standard_normal((1, T, H, D)), G, which, dtype, D ** -0.5)
    R.check(got, want, bound, kind)


@pytest.mark.parametrize("D,G,T,H,which,dtype", CASES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [160, 900, 3000])
def test_no_numbers(D, G, T, H, which, dtype, value, n):
    rng = np.random.default_rng(D + n)
    q = rng.standard_normal((1, T, H, D))
    clean = R.to_type(q, dtype, "cpu")[1]
    i, h = T // 2, H // 2
    q[0, i, h, D - 3] = value
    got, want, bound = run(rng, rng.standard_normal((n, 1, D)), rng.standard_normal((n, 1, D)), q, G, which, dtype, D ** -0.5,
                           qdef=clean)
    assert np.isnan(got[0, i, h]).all()
    keep = np.ones((T, H), bool)
    keep[i, h] = False
    R.check(got[0][keep], want[0][keep], bound[0][keep], "other rows")
