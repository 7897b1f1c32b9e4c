"""A window as large as an int holds is no limit, for sequences of fewer tokens than queries too."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 5, 2 ** 30])
@pytest.mark.parametrize("dtype,T,which", [("f32", 6, 1), ("bf16", 6, 1), ("f16", 90, 2)])
def test_widest_windows(window, dtype, T, which):
    rng = np.random.default_rng(T)
    lens = [3, T, T + 40, 0, T // 2]
    cache = R.Cache(rng, 5, lens, 2, 64, 32, 16)
    cache_t, table = cache.tensors(dev())
    q, _ = R.to_type(rng.standard_normal((5, T, 4, 64)), dtype, dev())
    c, n = fgq.KVCache(*cache_t), torch.tensor(lens, dtype=torch.int32, device=dev())
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        want = fgq.fgq_kv_attention(q, c, table, n)
        got = fgq.fgq_kv_attention(q, c, table, n, window=window)
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    assert got[0, -3:].any() and torch.equal(got, want)
