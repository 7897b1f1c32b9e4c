"""Sizes that the operators around the attention block refuse on the host, because a kernel would count past 32 bits."""
import ctypes

import pytest

from test_layer_host import L, P, w4  # noqa: F401


@pytest.mark.parametrize("rows", [2 ** 30 - 2 ** 15 + 1, 2 ** 30, 2 ** 31 - 2 ** 16 - 1])
def test_fp32_tokens_of_two_rows(L, rows):  # noqa: F811
    """Rows of two parts: twice the tokens, and a tile past them, have to be a 32-bit number."""
    from paper_1705_01462_gb300 import fgq
    assert L.fgq_linear_w4(P, 0, rows, 8, ctypes.byref(w4(rows=1, cols=8)), None, P, None) == fgq.FGQ_ERR_UNSUPPORTED
