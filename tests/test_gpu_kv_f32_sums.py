"""Sums of fp32 attention over many tokens carry no bias: each step of a sum is rounded to nearest, not cut off."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,Hq", [(64, 4), (128, 8)])
def test_no_bias(D, Hq):
    """Values of one sign, and so many sequences (sharing their pages) that one block takes thousands of tokens.  Roundings to
    nearest err to both sides, so that the mean over a thousand outputs keeps less than 2^-21; sums that are cut
    off lose half a unit in the last place, 2^-25 of the sum, in each of hundreds of steps."""
    rng = np.random.default_rng(D)
    n, B = 40000, 480
    cache = R.Cache(rng, 1, [n], 1, D, 64, 16)
    v = rng.uniform(1.4, 1.5, cache.v[0].shape).astype(np.float32)
    v[..., ::64] = 0.0  # so that the other codes of a group all lie on one side of its centre
    cache.v = R.quantize4(v, 64)
    cache.packed[2], cache.packed[3] = R.pack_codes(cache.v[0], False), R.pack_params(*cache.v[1:])
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(0.1 * rng.standard_normal((B, 1, Hq, D)), "f32", dev())
    out = fgq.fgq_kv_attention(q, fgq.KVCache(*cache_t), table.expand(B, -1).contiguous(),
                               torch.full((B,), n, dtype=torch.int32, device=dev()), max_len=n)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    got = out[:4].double().cpu().numpy()
    want = np.concatenate([R.attention(cache, qx[b:b + 1], [n], None, True, 0, D ** -0.5, "f32")[0] for b in range(4)])
    full = np.arange(D) % 64 != 0
    assert abs(np.mean(got[..., full] / want[..., full] - 1.0)) <= 2.0 ** -21
