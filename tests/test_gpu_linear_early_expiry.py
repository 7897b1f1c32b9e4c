"""Waits of the many-token product that run out anywhere in its course, in one block of a pair or in both: an error status, and the
next calls are right (no copy, commit or tensor memory is left behind)."""
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P,K,M", [(130, 4096, 260), (1000, 1024, 2048), (4100, 264, 2700)])
def test_limits_of_a_few_microseconds(P, K, M):
    g = torch.Generator(device=dev())
    g.manual_seed(P)
    x = torch.randn((P, K), generator=g, device=dev()).to(torch.bfloat16)
    w = torch.randint(-127, 128, (M, K), generator=g, device=dev(), dtype=torch.int8)
    s = torch.ones(M, device=dev())
    want = fgq.fgq_linear_w8a8(x, w, s)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    seen = set()
    for limit in (0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 40, 80):
        for _ in range(5):
            prev = fgq.fgq_debug_set_wait_limit_us(limit)
            try:
                y = fgq.fgq_linear_w8a8(x, w, s)
            finally:
                fgq.fgq_debug_set_wait_limit_us(prev)
            status = fgq.fgq_stream_status()
            assert status in (fgq.FGQ_OK, fgq.FGQ_ERR_TIMEOUT)
            assert status != fgq.FGQ_OK or torch.equal(y, want)
            seen.add(status)
            assert torch.equal(fgq.fgq_linear_w8a8(x, w, s), want)
            assert fgq.fgq_stream_status() == fgq.FGQ_OK
    assert seen == {fgq.FGQ_OK, fgq.FGQ_ERR_TIMEOUT}
