"""A linear layer whose output takes the place of its input gives what it gives elsewhere: no block may still read tokens where
another has written outputs."""
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("P,K", [(1, 4096), (4, 2048), (8, 1024), (40, 512), (200, 512)])
def test_output_over_the_input(P, K, dtype):
    g = torch.Generator(device=dev())
    g.manual_seed(P)
    w = torch.randint(-127, 128, (K, K), generator=g, device=dev(), dtype=torch.int8)
    s = torch.full((K,), 2.0 ** -10, device=dev())
    for _ in range(20):
        x = torch.randn((P, K), generator=g, device=dev()).to(dtype)
        want = fgq.fgq_linear_w8a8(x, w, s)
        assert fgq.fgq_linear_w8a8(x, w, s, y=x) is x and torch.equal(x, want)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_output_beside_the_input():
    """Rows of one buffer, input and output columns beside one another."""
    g = torch.Generator(device=dev())
    g.manual_seed(0)
    w = torch.randint(-127, 128, (64, 1024), generator=g, device=dev(), dtype=torch.int8)
    s = torch.ones(64, device=dev())
    buf = torch.randn(4 * 1024 + 64 * 4, generator=g, device=dev())
    x, y = buf[:4096].view(4, 1024), buf[4096:].view(4, 64)
    want = fgq.fgq_linear_w8a8(x.clone(), w, s)
    assert torch.equal(fgq.fgq_linear_w8a8(x, w, s, y=y), want)
