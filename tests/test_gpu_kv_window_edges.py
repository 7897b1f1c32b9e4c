"""Slots before a sliding window that share the window's first block of 16 tokens, or its page, with it may hold
anything: NaN and infinite parameters there must not reach the output."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("garbage", [0x7FC07FC0, 0x7F807F80, 0xFF80FF80])
@pytest.mark.parametrize("dtype,T", [("f32", 1), ("bf16", 1), ("bf16", 3), ("f16", 40), ("bf16", 150)])
@pytest.mark.parametrize("n,window", [(200, 30), (333, 70), (4116, 40)])
def test_garbage_before_the_window(dtype, T, n, window, garbage):
    rng = np.random.default_rng(n + T)
    D, G, page = 64, 32, 64
    cache = R.Cache(rng, 1, [n], 2, D, G, page)
    first = max(0, n - T + 1 - window)  # the first position that any query sees
    for i in (1, 3):
        for p in range(first):
            cache.packed[i][cache.table[0, p // page], :, p % page] = garbage
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((1, T, 4, D)), dtype, dev())
    out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, torch.tensor([n], dtype=torch.int32, device=dev()),
                               window=window)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, [n], None, True, window, D ** -0.5, dtype, fp16_rows=T > 16)
    R.check(out.float().cpu().numpy(), want, bound, "window")
