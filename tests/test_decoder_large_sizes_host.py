"""Sizes whose indices would pass 32 bits inside a kernel are refused on the host, before anything is launched."""
import pytest

from test_decoder_host import L, P, append, cache  # noqa: F401

TOP = 2 ** 31 - 1


@pytest.mark.parametrize("sizes", [dict(K=TOP), dict(K=TOP - 100), dict(rows=TOP), dict(M=TOP), dict(M=TOP - 30),
                                   dict(M=TOP, rows=100), dict(rows=TOP, K=0)])
def test_layers(L, sizes):  # noqa: F811
    from paper_1705_01462_gb300 import fgq
    rows, K, M = sizes.get("rows", 1), sizes.get("K", 1), sizes.get("M", 1)
    assert L.fgq_gemm_w8a8(P, P, rows, K, P, P, M, None, P, 0, None) == fgq.FGQ_ERR_UNSUPPORTED
    assert L.fgq_linear_w8a8(P, 0, rows, K, K, P, P, M, None, P, None) == fgq.FGQ_ERR_UNSUPPORTED
    if M == 1:
        assert L.fgq_quantize_tokens(P, 0, rows, K, K, P, P, None) == fgq.FGQ_ERR_UNSUPPORTED


@pytest.mark.parametrize("T", [TOP, TOP - 15])
def test_cache(L, T):  # noqa: F811
    from paper_1705_01462_gb300 import fgq
    c = cache(kv_heads=1)
    assert append(L, c, T=T) == fgq.FGQ_ERR_UNSUPPORTED
    assert L.fgq_kv_read(c[0], P, P, 0, 1, T, P, 4, P, None, None) == fgq.FGQ_ERR_UNSUPPORTED
