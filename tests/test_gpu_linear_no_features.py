"""Layers without input features give the bias, for any number of tokens."""
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [65, 65535 * 32, 65535 * 32 + 1, 65535 * 32 * 2 + 77])
def test_bias_alone(tokens):
    w = torch.empty((3, 0), dtype=torch.int8, device=dev())
    s = torch.ones(3, device=dev())
    bias = torch.tensor([1.0, -2.0, 0.5], device=dev())
    y = fgq.fgq_linear_w8a8(torch.empty((tokens, 0), device=dev()), w, s, bias=bias)
    assert torch.equal(y, bias.expand(tokens, 3))
    q = torch.empty((tokens, 0), dtype=torch.int8, device=dev())
    y = fgq.fgq_gemm_w8a8(q, torch.ones(tokens, device=dev()), w, s, bias=bias, dtype=torch.float16)
    assert torch.equal(y, bias.half().expand(tokens, 3))
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
