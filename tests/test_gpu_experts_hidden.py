"""What experts' outputs lose by how hidden values are held between the layers: less than their own rounding shows."""
import numpy as np
import pytest
import torch

import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_moe_w4 import layer

pytestmark = pytest.mark.gpu


# One token, units of one to eight tokens, units of 64 and 128 tokens; long rows.
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("P,K,F,E,top", [(1, 1024, 512, 16, 4), (9, 512, 768, 6, 2), (40, 512, 512, 20, 3), (60, 512, 512, 2, 1), (300, 512, 640, 4, 1),
                                         (5, 256, 9000, 3, 1)])
def test_outputs_round_as_exact_ones(dtype, P, K, F, E, top):
    """The distance to the definition in 64 bits rounded once, relative to the outputs' norm.

    An error of d of an output's magnitude takes it across a rounding's border with a probability of d / step and by a step then, so the
    distance is about sqrt(step d), step being at most 2 U of the value: 2^-7 (bf16), 2^-10 (fp16).  Hidden values are within 2^-22, sums'
    roundings and cut-offs below 2^-20 of the outputs' norm (a matrix instruction cuts off 2^-24 of its largest term or less, and they add up as
    independent ones do): d <= 2^-19, and sqrt(2^-7 2^-19) = 2^-13, sqrt(2^-10 2^-19) = 2^-14.5.  (Hidden values within 2^-12 would be at 2^-10.)
    Outputs of fp32: d itself."""
    rng = np.random.default_rng(P + F)
    on, d = layer(rng, E, K, F, 64)
    x, x64 = R.rng_tensor(rng, (P, K), dtype)
    ids = np.stack([rng.permutation(E)[:top] for _ in range(P)]).astype(np.int32)
    g = rng.random((P, top)).astype(np.float32)
    y = fgq.fgq_experts_w4(x.to(dev()), torch.from_numpy(ids).to(dev()), torch.from_numpy(g).to(dev()), *on)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    want, _ = R.experts(x64, ids, g.astype(np.float64), np.zeros((P, 1)), *d, 64, 64, dtype)
    once = torch.from_numpy(want).to(R.TYPES[dtype]).double().numpy()
    far = np.linalg.norm(y.double().cpu().numpy() - once) / np.linalg.norm(want)
    assert far <= {"bf16": 2.0 ** -13, "f16": 2.0 ** -14.5, "f32": 2.0 ** -19}[dtype], far
