"""Queries that hold NaN: their rows are NaN however the call is split and whichever kernel runs it, other
rows are within their bounds of the definition, and rows that see nothing stay zero."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu

# (tokens, max_len): one chunk, chunks that join as a cluster, through join_few_kernel (16 chunks at most) and
# join_kernel (more)
FORMS = [(20, 20), (700, 700), (5003, 5003), (60000, 60000)]


def call(n, max_len, dtype, spoiled, value, which=0, T=1, q_lens=None, D=64):
    """Output of one call (heads 4, kv heads 2) whose queries at `spoiled` hold `value` in places, with all rows but those
    checked against the definition."""
    rng = np.random.default_rng(n + T)
    cache = R.Cache(rng, 1, [n], 2, D, 64, 16)
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((1, T, 4, D)), dtype, dev())
    lens = torch.tensor([n], dtype=torch.int32, device=dev())
    nq = None if q_lens is None else torch.tensor([q_lens], dtype=torch.int32, device=dev())
    for i, h in spoiled:
        q[0, i, h, 7] = value
    prev = fgq.fgq_debug_set_attention_kernel(which)
    try:
        out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table, lens, q_lens=nq, max_len=max_len)
    finally:
        fgq.fgq_debug_set_attention_kernel(prev)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, bound = R.attention(cache, qx, [n], None if q_lens is None else [q_lens], True, 0, D ** -0.5, dtype,
                              fp16_rows=which == 2)
    keep = np.ones((T, 4), bool)
    for i, h in spoiled:
        keep[i, h] = q_lens is not None and i >= q_lens
    R.check(out[0].float().cpu().numpy()[keep], want[0][keep], bound[0][keep], "other rows")
    return out


@pytest.mark.parametrize("n,max_len", FORMS)
@pytest.mark.parametrize("dtype,which", [("f32", 1), ("bf16", 1), ("f16", 1), ("bf16", 2), ("f16", 2)])
def test_rows(n, max_len, dtype, which):
    out = call(n, max_len, dtype, [(0, 1)], float("nan"), which=which)
    assert out[0, 0, 1].isnan().all()


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,which", [("f32", 1), ("bf16", 1), ("f16", 2)])
def test_queries_that_do_not_exist(dtype, which, value):
    """Padding queries may hold anything: they give zeros."""
    out = call(300, 300, dtype, [(i, h) for i in (3, 4) for h in range(4)], value, which=which, T=5, q_lens=3)
    assert not out[0, 3:].any()
