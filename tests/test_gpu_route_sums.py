"""How exact logits are: runs of eight terms from the row's start are summed in fp32, and their sums as pairs of fp32."""
import numpy as np
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq


pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [24, 64, 512, 1001])
def test_terms_of_different_runs(K):
    """2^24 + 1 - 2^24 is 1, above 0.5, with the three terms in three runs."""
    rng = np.random.default_rng(K)
    x = torch.ones((3, K), device=dev())
    for _ in range(25):
        spots = 8 * rng.permutation(K // 8)[:3] + rng.integers(0, 8, 3)
        r = torch.zeros((5, K), device=dev())
        r[3, spots[0]], r[3, spots[1]], r[3, spots[2]] = 2.0 ** 24, 1.0, -2.0 ** 24
        r[1, spots[1]] = 0.5
        ids, w = fgq.fgq_route_tokens(x, r, 3)
        assert ids.tolist() == [[3, 1, 0]] * 3, spots
        want = np.exp([1.0, 0.5, 0.0])
        assert np.abs(w.double().cpu().numpy() - want / want.sum()).max() <= 2.0 ** -21


@pytest.mark.parametrize("dtype,rdtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("P,K", [(1, 8), (5, 13), (4, 1000), (9, 4096)])
def test_terms_of_one_run(dtype, rdtype, P, K):
    """Large terms that cancel beside small ones in the same run: logits are within 2^-21 of their terms' magnitudes, which is what the weights
    say: with an expert whose logit is exactly 0, their ratios are exponentials of the logits (each within 2^-21 of itself)."""
    rng = np.random.default_rng(K)
    E = 6
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    x = torch.from_numpy(rng.standard_normal((P, K)).astype(np.float32)).to(t[dtype])
    r = torch.from_numpy((rng.standard_normal((E, K)) / K ** 0.5).astype(np.float32)).to(t[rdtype])
    for k in range(0, K - 1, 8):  # +- pairs of terms 1000 times as large, whose sum is 0
        x[:, k + 1] = x[:, k]
        r[:, k] = torch.from_numpy((1000 * rng.standard_normal(E)).astype(np.float32)).to(t[rdtype])
        r[:, k + 1] = -r[:, k]
    r[0] = 0
    xd, rd = x.double().numpy(), r.double().numpy()
    logits, off = xd @ rd.T, 2.0 ** -21 * (np.abs(xd) @ np.abs(rd).T)
    ids, w = fgq.fgq_route_tokens(x.to(dev()), r.to(dev()), E, "softmax", False)
    ids, w = ids.cpu().numpy(), w.double().cpu().numpy()
    got = np.zeros((P, E))
    np.put_along_axis(got, ids, np.log(w), 1)
    assert np.all(np.abs(got - got[:, :1] - logits) <= off + 2.0 ** -20 + 2.0 ** -23 * np.abs(logits))
