"""What the operators around the attention block refuse on the host (no kernel launches), the rotary tables, and the 64-bit
definitions that the GPU tests use, against plain cases."""
import ctypes
import os
import shutil

import numpy as np
import pytest

import _layer as R


@pytest.fixture(scope="module")
def L():
    if shutil.which("nvcc") is None and not os.path.exists("/usr/local/cuda/bin/nvcc"):
        pytest.skip("nvcc not available")
    from paper_1705_01462_gb300 import build, fgq
    build.build()
    return fgq.load()


P = ctypes.c_void_p(4096)
ONE = ctypes.c_float(1.0)
NAN, INF = ctypes.c_float(float("nan")), ctypes.c_float(float("inf"))


def at(n):
    return ctypes.c_void_p(n)


def w4(experts=1, rows=8, cols=8, group=64, codes=4096, scales=4096):
    from paper_1705_01462_gb300 import fgq
    return fgq._W4Struct(codes, scales, experts, rows, cols, group)


def test_rope_refusals(L):
    from paper_1705_01462_gb300 import fgq

    def call(x=P, y=at(8192), ty=0, B=1, T=2, heads=2, D=8, xs=(32, 16), ys=(32, 16), rot=8, layout=0, table=P, mag=ONE,
             inverse=0, starts=P, lens=None):
        return L.fgq_rope(x, y, ty, B, T, heads, D, *xs, *ys, rot, layout, table, mag, inverse, starts, lens, None)

    for kw in (dict(x=None), dict(y=None), dict(table=None), dict(starts=None), dict(B=-1), dict(T=-1), dict(heads=-1), dict(ty=3),
               dict(rot=0), dict(rot=7), dict(rot=10), dict(layout=2), dict(inverse=2), dict(mag=NAN), dict(mag=INF),
               dict(y=P, ys=(32, 24))):
        assert call(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(x=at(4098)), dict(y=at(8194)), dict(table=at(4100)), dict(starts=at(4098)), dict(lens=at(4098)),
               dict(ty=1, x=at(4097))):
        assert call(**kw) == fgq.FGQ_ERR_ALIGN, kw
    for kw in (dict(B=1 << 16, T=1 << 15), dict(B=1 << 10, T=1 << 10, heads=1 << 11), dict(D=1 << 17), dict(heads=1 << 28)):
        assert call(**kw) == fgq.FGQ_ERR_UNSUPPORTED, kw
    for kw in (dict(B=0, x=None), dict(T=0, x=None), dict(heads=0, x=None)):
        assert call(**kw) == fgq.FGQ_OK, kw


def test_rope_table(L):
    from paper_1705_01462_gb300 import fgq
    t = (ctypes.c_uint64 * 8)()
    nan, inf = float("nan"), float("inf")
    ok = (16, 1e4, 3, 2.0, 4096.0, 1.0, 32.0)
    assert L.fgq_rope_table(*ok, t) == fgq.FGQ_OK
    for i, v in ((0, 0), (0, 3), (0, -2), (1, 1.0), (1, nan), (1, inf), (2, 4), (2, -1), (3, 0.5), (3, nan), (3, inf), (4, 0.0),
                 (4, nan), (5, 32.0), (5, nan), (6, inf)):
        bad = list(ok)
        bad[i] = v
        assert L.fgq_rope_table(*bad, t) == fgq.FGQ_ERR_ARG, (i, v)
    assert L.fgq_rope_table(*ok, None) == fgq.FGQ_ERR_ARG
    assert L.fgq_rope_table(16, 1e4, 0, nan, nan, nan, nan, t) == fgq.FGQ_OK  # plain tables look at none of the others
    for rot, base, kw in ((2, 1e4, {}), (64, 1e4, {}), (128, 5e5, dict(scaling="linear", factor=4.0)),
                          (80, 1e4, dict(scaling="base", factor=8.0)), (2, 1e4, dict(scaling="base", factor=8.0)),
                          (128, 1e4, dict(scaling="ramp", factor=8.0, length=4096.0)),
                          (128, 5e5, dict(scaling="ramp", factor=8.0, length=8192.0, low=1.0, high=4.0))):
        got = fgq.rope_table(rot, base, device="cpu", **kw).numpy().astype(np.float64)
        want = R.freqs(rot, base, **kw) / (2 * np.pi) * 2.0 ** 64
        # 64-bit powers and a few 64-bit products of either side
        assert np.all(np.abs(got - want) <= 1 + 2.0 ** -46 * want)


def test_norm_refusals(L):
    from paper_1705_01462_gb300 import fgq

    def call(x=P, ty=0, rows=2, K=8, ldx=8, post=None, gate=None, ldg=8, per=1, scale=ONE, r=P, rty=0, ldr=8, s=P, lds=8,
             pre=(4096, 4096, 1e-5, 0), y=P):
        keep = [None if n is None else fgq._NormStruct(*n) for n in (post, pre)]
        ref = [None if n is None else ctypes.byref(n) for n in keep]
        return L.fgq_add_norm(x, ty, rows, K, ldx, ref[0], gate, ldg, per, scale, r, rty, ldr, s, lds, ref[1], y, None)

    for kw in (dict(x=None), dict(rows=-1), dict(K=0), dict(ty=3), dict(rty=3), dict(ty=1, rty=2), dict(ty=0, rty=1), dict(ldx=7),
               dict(ldr=7), dict(lds=7), dict(gate=P, ldg=7), dict(gate=P, per=0), dict(scale=NAN), dict(scale=INF), dict(pre=None),
               dict(y=None), dict(pre=None, y=None, s=None), dict(pre=(4096, None, 0.0, 0)), dict(pre=(4096, None, float("nan"), 0)),
               dict(pre=(4096, None, 1e-5, 2)), dict(post=(4096, None, -1.0, 0)), dict(post=(4096, None, 1e-5, -1))):
        assert call(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(x=at(4098)), dict(r=at(4098)), dict(s=at(4098)), dict(y=at(4098)), dict(gate=at(4097), ty=1, rty=1),
               dict(pre=(4098, None, 1e-5, 0)), dict(post=(None, 4098, 1e-5, 1)), dict(ty=1, rty=0, r=at(4098))):
        assert call(**kw) == fgq.FGQ_ERR_ALIGN, kw
    big = 2 ** 31 - 1
    assert call(rows=big) == fgq.FGQ_ERR_UNSUPPORTED and call(K=big, ldx=big, ldr=big, lds=big) == fgq.FGQ_ERR_UNSUPPORTED
    assert call(rows=0, x=None) == fgq.FGQ_OK


def test_weight_refusals(L):
    from paper_1705_01462_gb300 import fgq
    q = lambda w=P, **kw: L.fgq_quantize_weights_w4(w, ctypes.byref(w4(**kw)), None)  # noqa: E731
    r = lambda o=P, **kw: L.fgq_read_weights_w4(ctypes.byref(w4(**kw)), o, None)  # noqa: E731
    for f in (q, r):
        for kw in (dict(rows=-1), dict(cols=-1), dict(experts=-1), dict(group=16), dict(group=256), dict(codes=None),
                   dict(scales=None)):
            assert f(**kw) == fgq.FGQ_ERR_ARG, kw
        assert f(None) == fgq.FGQ_ERR_ARG
        assert f(codes=4104) == fgq.FGQ_ERR_ALIGN and f(scales=4098) == fgq.FGQ_ERR_ALIGN and f(at(4098)) == fgq.FGQ_ERR_ALIGN
        assert f(rows=2 ** 31 - 1) == fgq.FGQ_ERR_UNSUPPORTED and f(cols=2 ** 31 - 1) == fgq.FGQ_ERR_UNSUPPORTED
        assert f(rows=1 << 20, cols=1 << 20, experts=4) == fgq.FGQ_ERR_UNSUPPORTED
        for kw in (dict(rows=0), dict(cols=0), dict(experts=0)):
            assert f(None, codes=None, **kw) == fgq.FGQ_OK, kw
    assert L.fgq_quantize_weights_w4(P, None, None) == fgq.FGQ_ERR_ARG
    assert L.fgq_w4_code_bytes(17, 129) == 4 * 1024 and L.fgq_w4_scale_bytes(17, 129, 32) == 4 * 16 * 4 * 2
    assert L.fgq_w4_code_bytes(-1, 5) == 0 and L.fgq_w4_scale_bytes(5, 5, 48) == 0 and L.fgq_w4_code_bytes(0, 5) == 0


def test_linear_refusals(L):
    from paper_1705_01462_gb300 import fgq

    def call(x=P, ty=0, rows=2, ldx=8, w=None, bias=None, y=P):
        return L.fgq_linear_w4(x, ty, rows, ldx, ctypes.byref(w or w4()), bias, y, None)

    for kw in (dict(x=None), dict(y=None), dict(ty=3), dict(rows=-1), dict(ldx=7), dict(w=w4(experts=2)), dict(w=w4(experts=0)),
               dict(w=w4(group=8)), dict(w=w4(codes=None))):
        assert call(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(x=at(4098)), dict(y=at(4098)), dict(bias=at(4098)), dict(ty=2, x=at(4097)), dict(w=w4(codes=4100))):
        assert call(**kw) == fgq.FGQ_ERR_ALIGN, kw
    assert call(rows=2 ** 31 - 1) == fgq.FGQ_ERR_UNSUPPORTED and call(w=w4(rows=1 << 25, cols=1 << 25), ldx=1 << 25) == fgq.FGQ_ERR_UNSUPPORTED
    assert call(rows=0, x=None) == fgq.FGQ_OK and call(w=w4(rows=0, codes=None), x=None) == fgq.FGQ_OK
    assert L.fgq_linear_w4(P, 0, 1, 8, None, None, P, None) == fgq.FGQ_ERR_ARG


def test_route_refusals(L):
    from paper_1705_01462_gb300 import fgq

    def call(x=P, ty=0, rows=2, K=8, ldx=8, router=P, rty=0, E=4, top=2, score=0, renorm=1, scale=ONE, ids=P, weights=P):
        return L.fgq_route_tokens(x, ty, rows, K, ldx, router, rty, E, top, score, renorm, scale, ids, weights, None)

    for kw in (dict(x=None), dict(router=None), dict(ids=None), dict(weights=None), dict(rows=-1), dict(K=0), dict(E=0), dict(ty=3),
               dict(ty=1, rty=2), dict(ty=0, rty=1), dict(top=0), dict(top=5), dict(score=2), dict(renorm=2), dict(scale=NAN),
               dict(ldx=7)):
        assert call(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in (dict(x=at(4098)), dict(router=at(4098)), dict(ids=at(4098)), dict(weights=at(4098))):
        assert call(**kw) == fgq.FGQ_ERR_ALIGN, kw
    for kw in (dict(E=1025), dict(E=64, top=33), dict(rows=2 ** 31 - 1), dict(K=2 ** 31 - 1, ldx=2 ** 31 - 1)):
        assert call(**kw) == fgq.FGQ_ERR_UNSUPPORTED, kw
    assert call(rows=0, x=None) == fgq.FGQ_OK


def test_experts_refusals(L):
    from paper_1705_01462_gb300 import fgq

    def parts(E=4, K=8, F=6, **kw):
        f = dict(gate=w4(E, F, K), up=w4(E, F, K), down=w4(E, K, F))
        f.update(kw)
        return [ctypes.byref(f[n]) for n in ("gate", "up", "down")]

    def call(x=P, ty=0, rows=2, ldx=8, ids=P, weights=P, top=2, y=P, **kw):
        return L.fgq_experts_w4(x, ty, rows, ldx, ids, weights, top, *parts(**kw), y, None)

    def layer(x=P, ty=0, rows=2, ldx=8, router=P, rty=0, top=2, score=0, renorm=1, scale=ONE, y=P, **kw):
        return L.fgq_moe_w4(x, ty, rows, ldx, router, rty, top, score, renorm, scale, *parts(**kw), y, None)

    both = (dict(x=None), dict(y=None), dict(ty=3), dict(rows=-1), dict(ldx=7), dict(top=0), dict(up=w4(4, 6, 9)), dict(up=w4(3, 6, 8)),
            dict(up=w4(4, 6, 8, group=32)), dict(up=w4(4, 5, 8)), dict(down=w4(4, 6, 8)), dict(down=w4(3, 8, 6)), dict(gate=w4(4, 6, 8, 7)),
            dict(F=0), dict(E=0))
    for kw in both + (dict(ids=None), dict(weights=None), dict(top=33)):
        assert call(**kw) == fgq.FGQ_ERR_ARG, kw
    for kw in both + (dict(router=None), dict(rty=3), dict(top=5), dict(score=-1), dict(renorm=3), dict(scale=INF)):
        assert layer(**kw) == fgq.FGQ_ERR_ARG, kw
    for f in (call, layer):
        for kw in (dict(x=at(4098)), dict(y=at(4098)), dict(gate=w4(4, 6, 8, codes=4100))):
            assert f(**kw) == fgq.FGQ_ERR_ALIGN, kw
        assert f(E=1025) == fgq.FGQ_ERR_UNSUPPORTED and f(rows=2 ** 31 - 1) == fgq.FGQ_ERR_UNSUPPORTED
        assert f(rows=0, x=None) == fgq.FGQ_OK
    assert call(ids=at(4098)) == fgq.FGQ_ERR_ALIGN and layer(router=at(4097)) == fgq.FGQ_ERR_ALIGN


def test_definitions_on_plain_cases():
    """Hand-checked: a quarter turn; a norm of equal values; codes of a group 0..7; the packing's word order; silu(0) = 0."""
    x = np.array([1.0, 2.0, 3.0, 4.0]).reshape(1, 1, 1, 4)
    y, _ = R.rope(x, np.array([np.pi / 2, 0.0]), [1], None, "half", 1.0, False, "f32")
    assert np.allclose(y.ravel(), [-3, 2, 1, 4])
    y, _ = R.rope(x, np.array([np.pi / 2, np.pi]), [1], None, "interleaved", 2.0, True, "f32")
    assert np.allclose(y.ravel(), [4, -2, -6, -8])
    y, e = R.norm(np.array([[3.0, 4.0]]), np.zeros((1, 2)), None, None, "rms", 0.0)
    assert np.allclose(y, np.array([3, 4]) / np.sqrt(12.5)) and np.all(e < 1e-5)
    y, _ = R.norm(np.array([[1.0, 3.0]]), np.zeros((1, 2)), np.array([2.0, 2.0]), np.array([1.0, 0.0]), "layer", 0.0)
    assert np.allclose(y, [[-1, 2]])
    c, s = R.quantize_w4(np.arange(32, dtype=np.float32)[None] % 8, 32)
    assert s[0, 0] == 1 and np.array_equal(c[0], np.arange(32) % 8)
    rng = np.random.default_rng(0)
    c, s = R.random_w4(rng, (2, 21, 300), 64)
    codes, sc = R.pack_w4(c, s, 64)
    assert codes.shape == (2, 2, 3, 1024) and sc.shape == (2, 2, 3, 16, 2)
    assert np.array_equal(R.unpack_w4(codes, 21, 300), c)
    word = codes[0, 0, 0].view(np.uint32)  # row 1, columns 40 .. 47: g = 1, r = 0, t = 1, j = 1
    nib = [int(word[(1 * 4 + 1) * 4 + 1] >> (4 * n) & 15) - 8 for n in (0, 4, 1, 5, 2, 6, 3, 7)]
    assert nib == c[0, 1, 40:48].tolist()
    assert sc[1, 1, 2, 4, 0] == s[1, 20, 4].view(np.uint32) >> 16
    ids, g, _ = R.route(np.ones((1, 1)), np.array([[1.0], [2.0], [2.0], [0.0]]), 3, "softmax", True, 2.0)
    assert ids.tolist() == [[1, 2, 0]] and np.isclose(g.sum(), 2)
    w = np.ones((1, 2, 2))
    y, _ = R.experts(np.array([[1.0, -1.0]]), np.array([[0, -1]]), np.ones((1, 2)), np.zeros((1, 1)), w, w, w, 32, 32, "f32")
    assert np.all(y == 0)
