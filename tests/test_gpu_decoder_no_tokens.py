"""A decoder block called without tokens: for all sequences, or for some."""
import pytest

from paper_1705_01462_gb300 import fgq
from test_gpu_decoder_release import fresh

pytestmark = pytest.mark.gpu


def test_no_tokens():
    b, x = fresh()
    assert b.forward(x[:, :0]).shape == (2, 0, 96)
    b.forward(x[:, :3])
    assert b.forward(x[:, :0]).shape == (2, 0, 96) and b.lengths == [3, 3]
    y = b.forward(x[:, :2], lens=[0, 0])
    assert y.shape == (2, 2, 96) and b.lengths == [3, 3]
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
