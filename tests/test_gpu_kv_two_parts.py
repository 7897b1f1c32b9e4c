"""fp16 outputs of the kernel for many query rows take probabilities as two fp16 parts: cases in which a probability's rounding is
all that is left but the output's own, and one part alone would show."""
import numpy as np
import pytest
import torch

import _decoder as R
import _kv_content as C

N, T = 200, 150


def case(D, rng):
    """Keys with 0 .. 15 in one place (exact, as their group spans 0 .. 15), values 15 in one of sixteen places: output d of a
    query is 15 times the probability that falls on the tokens of key d."""
    c = np.arange(N) % 16
    k, v = np.zeros((N, 1, D)), np.zeros((N, 1, D))
    k[:, 0, 0], k[:, 0, 1] = c, 15
    v[np.arange(N), 0, c] = 15
    q = np.zeros((1, T, 1, D), np.float16)
    q[0, :, 0, 0] = rng.uniform(-1.2, 1.2, T)
    z = q[0, :, 0, :1].astype(np.float64) * c / 8  # the scale
    return k, v, q, z, c


def outputs(z, c, parts):
    """fp64 outputs of probabilities 64 2^x, x <= 0, of `parts` fp16 parts (0: exact), over their exact sum."""
    p = 64 * np.exp(z - z.max(1, keepdims=True))
    w = p
    if parts:
        w = p.astype(np.float16).astype(np.float64)
        if parts == 2:
            w += (p - w).astype(np.float16).astype(np.float64)
    return 15 * np.stack([w[:, c == d].sum(1) for d in range(16)], 1) / p.sum(1, keepdims=True)


def outside(got, want):
    """Outputs further off than half an fp16 step and 2^-16 of the output: scores below 5 in log2 units by products and a sum
    that round to 2^-24, exponentials to 2^-22, second parts to 2^-22, and sums of 200 terms to 2^-24 each are below 2^-17."""
    half = 2.0 ** (np.maximum(np.floor(np.log2(want)), -14) - 11)
    return np.abs(got - want) > half + 2.0 ** -16 * want


def test_one_part_would_show():
    _, _, _, z, c = case(64, np.random.default_rng(1))
    want = outputs(z, c, 0)
    assert outside(outputs(z, c, 1).astype(np.float16).astype(np.float64), want).mean() > 0.1
    assert not outside(outputs(z, c, 2).astype(np.float16).astype(np.float64), want).any()


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [T, 100])  # two tiles of 128 rows, and one
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 64), (128, 128), (256, 32)])
def test_outputs(D, G, rows):
    from _gpu import dev
    from paper_1705_01462_gb300 import fgq
    rng = np.random.default_rng(1)
    k, v, q, z, c = case(D, rng)
    cache = C.cache_of(rng, k, v, G)
    cache_t, table = cache.tensors(dev())
    assert fgq.fgq_debug_set_attention_kernel(2) == 0
    try:
        out = fgq.fgq_kv_attention(torch.from_numpy(q[:, :rows]).to(dev()), fgq.KVCache(*cache_t), table,
                                   torch.tensor([N], dtype=torch.int32, device=dev()), causal=False, scale=0.125)
    finally:
        fgq.fgq_debug_set_attention_kernel(0)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    got = out[0, :, 0].double().cpu().numpy()
    bad = outside(got[:, :16], outputs(z, c, 0)[:rows])
    assert not bad.any(), f"{bad.sum()} of {bad.size}"
    assert not got[:, 16:].any()
