"""Outputs of the operators around the attention block that would overwrite one another, or inputs of other tokens, are refused on the host."""
import ctypes

import pytest

from test_layer_host import L, ONE, P, at  # noqa: F401


@pytest.mark.parametrize("B,T,bs,ts", [(1, 2, 0, 0), (1, 2, 0, 15), (3, 1, 0, 0), (3, 1, 15, 0), (2, 3, 16, 16), (2, 3, 47, 16), (2, 3, 0, 16), (3, 2, 16, 47),
                                       (2, 3, -16, 16), (2, 3, 40, 20), (1 << 10, 1 << 10, 1 << 10, 1 << 10)])
def test_rope_tokens_that_overlap(L, B, T, bs, ts):  # noqa: F811
    from paper_1705_01462_gb300 import fgq
    for y in (P, at(1 << 20)):
        assert L.fgq_rope(P, y, 0, B, T, 2, 8, bs, ts, bs, ts, 8, 0, P, ONE, 0, P, None, None) == fgq.FGQ_ERR_ARG


@pytest.mark.parametrize("kw", [dict(x=P, y=P, ldx=9), dict(x=P, y=P, ldx=16), dict(r=P, s=P, ldr=8, lds=9), dict(r=P, s=P, ldr=16, lds=8)])
def test_norm_rows_that_overlap(L, kw):  # noqa: F811
    from paper_1705_01462_gb300 import fgq
    a = dict(x=at(1 << 20), y=at(2 << 20), r=at(3 << 20), s=at(4 << 20), ldx=8, ldr=8, lds=8)
    a.update(kw)
    n = fgq._NormStruct(None, None, 1e-5, 0)
    assert L.fgq_add_norm(a["x"], 0, 2, 8, a["ldx"], None, None, 0, 0, ONE, a["r"], 0, a["ldr"], a["s"], a["lds"], ctypes.byref(n), a["y"],
                          None) == fgq.FGQ_ERR_ARG
