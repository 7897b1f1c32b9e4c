"""Sizes past 32 bits are refused, not cut off to what their lower bits say.  (Tensors of one element's memory stand for them.)"""
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu

BIG = [2 ** 31, 2 ** 32 + 3]


def refused(call):
    with pytest.raises(fgq.FGQError) as e:
        call()
    assert e.value.code == fgq.FGQ_ERR_UNSUPPORTED


@pytest.mark.parametrize("n", BIG)
def test_sizes(n):
    one = lambda *shape: torch.zeros((1,) * len(shape), device=dev(), dtype=torch.bfloat16).expand(shape)  # noqa: E731
    starts, table = torch.zeros(1, dtype=torch.int32, device=dev()), fgq.rope_table(2, device=dev())
    for shape in ((n, 1, 1, 2), (1, n, 1, 2), (1, 1, n, 2), (1, 1, 1, n)):
        refused(lambda: fgq.fgq_rope(one(*shape), table, starts))
    refused(lambda: fgq.fgq_rope(one(1, 1, 1, 2), torch.zeros(1, dtype=torch.int64, device=dev()).expand(n // 2), starts))
    refused(lambda: fgq.rope_table(n, device=dev()))
    norm = fgq.Norm()
    refused(lambda: fgq.fgq_add_norm(one(n, 1), None, norm))
    refused(lambda: fgq.fgq_add_norm(one(1, n)[:, :1].expand(n, 1), one(n, 1), norm))
    refused(lambda: fgq.fgq_quantize_weights_w4(torch.zeros((1, 1), device=dev()).expand(n, 1)))
    w = fgq.fgq_quantize_weights_w4(torch.zeros((1, 1, 1), device=dev()))
    refused(lambda: fgq.fgq_linear_w4(one(n, 1), w))
    x, r = one(1, 1), one(1, 1)
    refused(lambda: fgq.fgq_route_tokens(one(n, 1), r, 1))
    refused(lambda: fgq.fgq_route_tokens(x, r, n))
    refused(lambda: fgq.fgq_moe_w4(one(n, 1), r, 1, w, w, w))
    refused(lambda: fgq.fgq_moe_w4(x, r, n, w, w, w))
    refused(lambda: fgq.fgq_moe_w4(x, r, n + 1, w, w, w))
