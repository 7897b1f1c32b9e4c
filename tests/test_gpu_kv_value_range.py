"""Values of all magnitudes that the cache is stated to serve, groups of equal values (whose scale is 0) among them, on both
attention kernels."""
import numpy as np
import pytest
import torch

import _decoder as R
import _kv_content as C
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def check(rng, v, dtype, which, T=1, Hq=2, G=32):
    n, Hkv, D = v.shape
    cache = C.cache_of(rng, rng.standard_normal((n, Hkv, D)), v, G)
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((1, T, Hq, D)), dtype, dev())
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()))
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, [n], None, True, 0, D ** -0.5, dtype, fp16_rows=which == 2)
    R.check(out.float().cpu().numpy(), want, bound, "values")


KERNELS = [("f32", 1), ("bf16", 1), ("bf16", 2)]


@pytest.mark.parametrize("n", [1, 100, 700])
@pytest.mark.parametrize("value", [1e-3, -1.0, 2.0 ** 67, -1.5 * 2.0 ** 99])
@pytest.mark.parametrize("dtype,which", KERNELS)
def test_equal_values(n, value, dtype, which):
    """(The larger ones bf16 values, so that the scale is 0.)"""
    check(np.random.default_rng(n), np.full((n, 1, 64), value), dtype, which)


@pytest.mark.parametrize("value", [2.0 ** 67, -1.5 * 2.0 ** 99])
@pytest.mark.parametrize("at", [0, 70, 200, 699])
@pytest.mark.parametrize("dtype,which", KERNELS)
def test_one_group_that_varies(value, at, dtype, which):
    """One token's values vary, in one warp's tile or chunk; all others are equal."""
    rng = np.random.default_rng(at)
    v = np.full((700, 1, 64), value)
    v[at] *= rng.uniform(0.5, 1.5, (1, 64))
    check(rng, v, dtype, which)


@pytest.mark.parametrize("magnitude", [1e-18, 1e-6, 1e25, 1e30])
@pytest.mark.parametrize("zeros", ["none", "first", "last", "most"])
@pytest.mark.parametrize("dtype,which", KERNELS)
def test_magnitudes_beside_zeros(magnitude, zeros, dtype, which):
    """Tokens whose values are all 0 weigh in the softmax as any other, whatever the rest's magnitude."""
    rng = np.random.default_rng(len(zeros))
    v = rng.standard_normal((700, 1, 64)) * magnitude
    v[{"none": slice(0, 0), "first": slice(0, 350), "last": slice(350, 700), "most": slice(0, 690)}[zeros]] = 0.0
    check(rng, v, dtype, which)
