"""The tests of long runs of queries and of a window's edges once more with the kernel for many query rows forced, which
small calls do not choose by themselves; single tokens on it; and both kernels side by side."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_kv_attention import run
from test_gpu_kv_prompt import *  # noqa: F401,F403
from test_gpu_kv_window_edges import test_garbage_before_the_window as window_edge

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def many_rows():
    assert fgq.fgq_debug_set_attention_kernel(2) == 0
    yield
    assert fgq.fgq_debug_set_attention_kernel(0) == 2


@pytest.mark.parametrize("T", [1, 2, 9])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_single_tokens(D, T):
    run(np.random.default_rng(T + D), 3, T, 8, 2, D, 64, 16, "bf16", [T, 0, T + 200], fp16_rows=True)


@pytest.mark.parametrize("garbage", [0x7FC07FC0, 0xFF80FF80])
@pytest.mark.parametrize("dtype,T", [("f16", 40), ("bf16", 150)])
@pytest.mark.parametrize("n,window", [(200, 30), (333, 70), (4116, 40)])
def test_window_edges(dtype, T, n, window, garbage):
    window_edge(n=n, window=window, dtype=dtype, T=T, garbage=garbage)


def test_other_values_are_refused():
    for which in (-1, 3):
        assert fgq.fgq_debug_set_attention_kernel(which) == -1


@pytest.mark.parametrize("T,Hq,Hkv,D", [(6, 8, 2, 64), (40, 4, 2, 128), (33, 3, 1, 256), (150, 2, 1, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_both_kernels_agree(T, Hq, Hkv, D, dtype):
    """Each is within its own bound of the definition, so the two are within the sum."""
    rng = np.random.default_rng(T)
    n = [T + 130, T]
    cache = R.Cache(rng, 2, n, Hkv, D, 64, 16)
    cache_t, table = cache.tensors(dev())
    q, qx = R.to_type(rng.standard_normal((2, T, Hq, D)), dtype, dev())
    args = (q, fgq.KVCache(*cache_t), table, torch.tensor(n, dtype=torch.int32, device=dev()))
    many = fgq.fgq_kv_attention(*args).float().cpu().numpy()
    assert fgq.fgq_debug_set_attention_kernel(1) == 2
    few = fgq.fgq_kv_attention(*args).float().cpu().numpy()
    assert fgq.fgq_debug_set_attention_kernel(2) == 1
    bounds = [R.attention(cache, qx, n, None, True, 0, D ** -0.5, dtype, fp16_rows=f)[1] for f in (False, True)]
    R.check(many, few.astype(np.float64), bounds[0] + bounds[1], "kernels")
