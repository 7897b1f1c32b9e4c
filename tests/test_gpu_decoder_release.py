"""A decoder block's sequences end, and others take their places."""
import pytest
import torch

from _gpu import dev
from paper_1705_01462_gb300 import fgq
from test_gpu_decoder import block

pytestmark = pytest.mark.gpu


def fresh(seed=7):
    b, g = block(seed, 96, 4, 2, 64, 32, 16, 8, 2)
    return b, torch.randn((2, 70, 96), generator=g, device=dev())


@pytest.mark.parametrize("how", ["block", "pool"])
def test_a_released_sequence_is_over(how):
    """A new prompt in the place of a released sequence gives what it gives in a fresh block: nothing of what its pages
    held before."""
    b, x = fresh()
    b.forward(x[:, :50], lens=[50, 20])
    (b.release if how == "block" else b.pool.release)(0)
    assert b.lengths == [0, 20]
    got = b.forward(x[:, 50:], lens=[20, 0])
    assert fgq.fgq_stream_status() == fgq.FGQ_OK and b.lengths == [20, 20]
    f, _ = fresh()
    want = f.forward(x[:, 50:], lens=[20, 0])
    assert torch.equal(got[0, :20], want[0, :20])
    # and the sequence that stayed goes on as if nothing had happened
    got = b.forward(x[:, :1], lens=[0, 1])[1, 0]
    g, _ = fresh()
    g.forward(x[:, :50], lens=[0, 20])
    assert torch.equal(got, g.forward(x[:, :1], lens=[0, 1])[1, 0])


def test_release_makes_room():
    b, x = fresh()  # eight pages of 16
    b.forward(x[:, :64], lens=[64, 60])
    with pytest.raises(RuntimeError):
        b.forward(x[:, :16], lens=[16, 0])
    assert b.lengths == [64, 60]
    b.release(1)
    b.forward(x[:, :16], lens=[16, 0])
    assert b.lengths == [80, 0]
