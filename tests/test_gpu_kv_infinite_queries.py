"""Queries that hold an infinity: their rows are NaN, as no softmax of their scores is defined, and not zeros where all
scores are the same negative infinity."""
import numpy as np
import pytest
import torch

import _decoder as R
import _kv_content as C
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_kv_nonfinite import FORMS, call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
@pytest.mark.parametrize("n,max_len", FORMS)
@pytest.mark.parametrize("dtype,which", [("f32", 1), ("bf16", 1), ("f16", 1), ("bf16", 2), ("f16", 2)])
def test_rows(n, max_len, dtype, which, value):
    out = call(n, max_len, dtype, [(0, 1)], value, which=which)
    assert out[0, 0, 1].isnan().all()


@pytest.mark.parametrize("dtype,which,T", [("f32", 1, 1), ("bf16", 1, 1), ("bf16", 2, 1), ("f16", 2, 40)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf")])
def test_keys_of_one_sign(dtype, which, T, value):
    rng = np.random.default_rng(T)
    n, D = 90, 64
    k = rng.uniform(1.0, 2.0, (n, 1, D))  # codes and parameters all positive
    cache = C.cache_of(rng, k, rng.standard_normal((n, 1, D)), 32)
    cache_t, table = cache.tensors(dev())
    q = torch.zeros((1, T, 2, D), dtype=R.TYPES[dtype], device=dev())
    q[0, 0, 1, 5] = value
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()))
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert out[0, 0, 1].isnan().all() and not out[0, 0, 0].isnan().any()
