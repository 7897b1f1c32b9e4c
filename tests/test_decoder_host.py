"""What the decoder operators refuse on the host (no kernel launches), and the 64-bit definitions that their GPU
tests use, against plain cases."""
import ctypes
import shutil
import os

import numpy as np
import pytest

import _decoder as R


@pytest.fixture(scope="module")
def L():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_1705_01462_gb300 import build, fgq
    build.build()
    return fgq.load()


P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4104)
F = ctypes.c_float(0.125)


def cache(**kw):
    from paper_1705_01462_gb300 import fgq
    f = dict(k_codes=4096, k_params=4096, v_codes=4096, v_params=4096, pages=4, page_size=16, kv_heads=2, head_dim=64,
             group=32)
    f.update(kw)
    c = fgq._KVCacheStruct(*(f[n] for n, _ in fgq._KVCacheStruct._fields_))
    return ctypes.addressof(c), c


def append(L, c, k=P, v=P, ty=0, B=1, T=4, strides=(512, 128, 512, 128), table=P, mp=4, starts=P, lens=None):
    return L.fgq_kv_append(c[0], k, v, ty, B, T, *strides, table, mp, starts, lens, None)


def attend(L, c, q=P, ty=0, B=1, T=2, heads=4, qbs=512, qts=256, table=P, mp=4, lens=P, q_lens=None, max_len=0,
           causal=1, window=0, scale=F, out=P):
    return L.fgq_kv_attention(c[0], q, ty, B, T, heads, qbs, qts, table, mp, lens, q_lens, max_len, causal, window,
                              scale, out, None)


def test_cache_refusals(L):
    from paper_1705_01462_gb300 import fgq
    for kw in (dict(k_codes=None), dict(v_params=None), dict(pages=0), dict(page_size=24), dict(page_size=0),
               dict(kv_heads=0), dict(head_dim=96), dict(group=16), dict(group=128)):
        assert append(L, cache(**kw)) == fgq.FGQ_ERR_ARG, kw
        assert attend(L, cache(**kw)) == fgq.FGQ_ERR_ARG, kw
    assert L.fgq_kv_append(None, P, P, 0, 1, 1, 128, 128, 128, 128, P, 1, P, None, None) == fgq.FGQ_ERR_ARG
    assert append(L, cache(k_params=4100)) == fgq.FGQ_ERR_ALIGN


def test_append_and_read_refusals(L):
    from paper_1705_01462_gb300 import fgq
    c = cache()
    for kw in (dict(k=None), dict(table=None), dict(starts=None), dict(B=-1), dict(T=-1), dict(ty=3), dict(mp=-1)):
        assert append(L, c, **kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(v=ODD), dict(strides=(514, 128, 512, 128)), dict(strides=(512, 128, 512, 129)),
               dict(starts=ctypes.c_void_p(4097)), dict(lens=ctypes.c_void_p(4098)), dict(ty=1, strides=(512, 124, 512, 128))):
        assert append(L, c, **kw) == fgq.FGQ_ERR_ALIGN, kw
    assert append(L, c, B=0, k=None) == fgq.FGQ_OK and append(L, c, T=0, k=None) == fgq.FGQ_OK
    assert append(L, cache(kv_heads=1 << 20), T=1 << 12) == fgq.FGQ_ERR_UNSUPPORTED
    assert L.fgq_kv_read(c[0], P, ODD, 0, 1, 4, P, 4, P, None, None) == fgq.FGQ_ERR_ALIGN
    assert L.fgq_kv_read(c[0], P, P, 5, 1, 4, P, 4, P, None, None) == fgq.FGQ_ERR_ARG


def test_attention_refusals(L):
    from paper_1705_01462_gb300 import fgq
    c = cache()
    for kw in (dict(q=None), dict(out=None), dict(table=None), dict(lens=None), dict(B=-1), dict(T=-1), dict(heads=5),
               dict(heads=0), dict(ty=9), dict(window=-1), dict(window=3, causal=0), dict(causal=2), dict(max_len=-1),
               dict(scale=ctypes.c_float(float("nan"))), dict(scale=ctypes.c_float(0.0)),
               dict(scale=ctypes.c_float(float("inf")))):
        assert attend(L, c, **kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(q=ODD), dict(out=ODD), dict(qts=255), dict(ty=2, qbs=516), dict(lens=ctypes.c_void_p(4097)),
               dict(q_lens=ctypes.c_void_p(4098))):
        assert attend(L, c, **kw) == fgq.FGQ_ERR_ALIGN, kw
    assert attend(L, c, B=0, q=None) == fgq.FGQ_OK and attend(L, c, T=0, q=None) == fgq.FGQ_OK
    assert attend(L, c, T=1 << 30, heads=4) == fgq.FGQ_ERR_UNSUPPORTED


def test_linear_refusals(L):
    from paper_1705_01462_gb300 import fgq
    quant = lambda x=P, ty=0, rows=2, K=8, ldx=8, q=P, s=P: L.fgq_quantize_tokens(x, ty, rows, K, ldx, q, s, None)  # noqa: E731
    for kw in (dict(x=None), dict(q=None), dict(s=None), dict(rows=-1), dict(K=-1), dict(ldx=7), dict(ty=-1)):
        assert quant(**kw) == fgq.FGQ_ERR_ARG, kw
    assert quant(x=ctypes.c_void_p(4098)) == fgq.FGQ_ERR_ALIGN and quant(s=ctypes.c_void_p(4098)) == fgq.FGQ_ERR_ALIGN
    assert quant(rows=0, x=None) == fgq.FGQ_OK
    gemm = lambda q=P, s=P, rows=2, K=8, w=P, ws=P, M=3, b=None, y=P, ty=0: L.fgq_gemm_w8a8(  # noqa: E731
        q, s, rows, K, w, ws, M, b, y, ty, None)
    for kw in (dict(q=None), dict(s=None), dict(w=None), dict(ws=None), dict(y=None), dict(rows=-1), dict(K=-1),
               dict(M=-1), dict(ty=3)):
        assert gemm(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(s=ctypes.c_void_p(4097)), dict(ws=ctypes.c_void_p(4098)), dict(b=ctypes.c_void_p(4098)),
               dict(y=ctypes.c_void_p(4098)), dict(y=ctypes.c_void_p(4097), ty=1)):
        assert gemm(**kw) == fgq.FGQ_ERR_ALIGN, kw
    assert gemm(rows=0, q=None) == fgq.FGQ_OK and gemm(M=0, w=None) == fgq.FGQ_OK
    lin = lambda x=P, ty=0, rows=2, K=8, ldx=8, w=P, ws=P, M=3, y=P: L.fgq_linear_w8a8(  # noqa: E731
        x, ty, rows, K, ldx, w, ws, M, None, y, None)
    for kw in (dict(x=None), dict(ldx=7), dict(w=None), dict(y=None), dict(ty=4), dict(M=-2)):
        assert lin(**kw) == fgq.FGQ_ERR_ARG, kw
    assert lin(x=ctypes.c_void_p(4098)) == fgq.FGQ_ERR_ALIGN
    assert lin(rows=0, x=None) == fgq.FGQ_OK


def test_definitions_on_plain_cases():
    """Hand-checked: a group 0..15 holds itself; rounding outwards; every nibble used once; the softmax bound's value."""
    x = np.tile(np.arange(32, dtype=np.float32) % 16, (1, 2))
    c, lo, s = R.quantize4(x, 32)
    assert np.array_equal(c, x.astype(np.uint8)) and not lo.any() and np.all(s == 1)
    v = np.float32(1.0) + np.float32(2.0 ** -9)
    assert R.bf16_round(v, True) == np.float32(1.0 + 2.0 ** -7) and R.bf16_round(v, False) == 1.0
    assert R.bf16_round(-v, False) == np.float32(-1.0 - 2.0 ** -7) and R.bf16_round(-v, True) == -1.0
    for D in (64, 128, 256):
        for keys in (True, False):
            assert sorted(R.nibble_of(d, D, keys) for d in range(D)) == list(range(D))
            codes = np.random.default_rng(0).integers(0, 16, (3, D)).astype(np.uint8)
            assert np.array_equal(R.unpack_codes(R.pack_codes(codes, keys), keys), codes)
    q, scale = R.quantize8(np.array([[0, 0], [1, -2], [63.5, 127]]))
    assert np.array_equal(q, [[0, 0], [64, -127], [64, 127]]) and scale[2] == 1
    rng = np.random.default_rng(1)
    cache = R.Cache(rng, 1, [9], 1, 64, 64, 16)
    qv = rng.standard_normal((1, 2, 1, 64))
    out, bound = R.attention(cache, qv, [9], None, True, 0, 0.125, "f32")
    k, v, _, _ = cache.rows(0, 9)
    z = k[0, :8] @ qv[0, 0, 0] * 0.125
    assert np.allclose(out[0, 0, 0], np.exp(z) @ v[0, :8] / np.exp(z).sum(), rtol=1e-12) and np.all(bound > 0)
