"""The 4-bit cache: what fgq_kv_append writes, bit for bit, and what fgq_kv_read gives back."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import fgq

pytestmark = pytest.mark.gpu


def table_for(rng, ends, page, extra=2):
    per = [max(1, -(-int(e) // page)) for e in ends]
    order = rng.permutation(sum(per) + extra).astype(np.int32)
    t = np.full((len(per), max(per)), -1, np.int32)
    at = 0
    for b, n in enumerate(per):
        t[b, :n] = order[at:at + n]
        at += n
    return t, sum(per) + extra


def written(x, table, starts, lens, pages, G, keys):
    """The packed cache after the call on an empty one, and the values that it then holds."""
    B, T, H, D = x.shape
    page = written.page
    codes = np.zeros((pages, H, page, D // 2), np.uint8)
    params = np.zeros((pages, H, page, D // G), np.uint32)
    c, lo, s = R.quantize4(x, G)
    back = R.dequantize4(c, lo, s)
    pc, pp = R.pack_codes(c, keys), R.pack_params(lo, s)
    for b in range(B):
        for i in range(T):
            if i >= lens[b]:
                back[b, i] = 0
                continue
            p = starts[b] + i
            codes[table[b, p // page], :, p % page] = pc[b, i]
            params[table[b, p // page], :, p % page] = pp[b, i]
    return codes, params, back


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,G", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128), (256, 32), (256, 64), (256, 128)])
def test_append_and_read(dtype, D, G):
    rng = np.random.default_rng(D + G)
    B, T, H, page = 3, 21, 3, 16
    starts, lens = np.array([0, 13, 40]), np.array([21, 1, 17])
    table, pages = table_for(rng, starts + lens, page)
    written.page = page
    cache = fgq.kv_cache(pages, page, H, D, G)
    xs = [rng.standard_normal((B, T, H, D)) * np.exp(rng.uniform(-3, 3, (B, T, H, 1))) for _ in "kv"]
    xs[0][0, 3] = 0.0          # a constant group: s = 0
    xs[0][0, 4] = -1.25
    xs[1][0, 5, :, ::2] = -0.0
    (kt, kx), (vt, vx) = (R.to_type(x, dtype, dev()) for x in xs)
    dt = torch.from_numpy(table).to(dev())
    st, ln = (torch.from_numpy(a.astype(np.int32)).to(dev()) for a in (starts, lens))
    fgq.fgq_kv_append(cache, kt, vt, dt, st, lens=ln)
    k, v = fgq.fgq_kv_read(cache, dt, st, T, lens=ln, dtype=torch.float32)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    for x, got, codes, params, keys in ((kx, k, cache.k_codes, cache.k_params, True),
                                        (vx, v, cache.v_codes, cache.v_params, False)):
        wc, wp, back = written(x.astype(np.float32), table, starts, lens, pages, G, keys)
        assert np.array_equal(params.cpu().numpy().view(np.uint32), wp)
        assert np.array_equal(codes.cpu().numpy(), wc)
        assert np.array_equal(got.cpu().numpy(), back.astype(np.float32))
    k16, _ = fgq.fgq_kv_read(cache, dt, st, T, lens=ln, dtype=torch.bfloat16)
    assert torch.equal(k16, k.to(torch.bfloat16))


def test_half_step_bound():
    """|x - (lo + s c)| is at most half a step (and the rounding of the fp32 difference and quotient)."""
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((1, 64, 2, 128)) * 3).astype(np.float32)
    cache = fgq.kv_cache(4, 16, 2, 128, 32)
    table = torch.arange(4, dtype=torch.int32, device=dev())[None]
    t = torch.from_numpy(x).to(dev())
    zero = torch.zeros(1, dtype=torch.int32, device=dev())
    fgq.fgq_kv_append(cache, t, t, table, zero)
    k, v = fgq.fgq_kv_read(cache, table, zero, 64, dtype=torch.float32)
    _, _, s = R.quantize4(x, 32)
    step = np.repeat(s, 32, -1).reshape(x.shape)
    for got in (k, v):
        assert np.all(np.abs(got.cpu().numpy() - x) <= step * (0.5 + 2e-6) + 1e-6)


def test_strided_inputs_and_another_stream():
    """Keys and values as views of one fused projection, on a stream of their own."""
    rng = np.random.default_rng(7)
    B, T, H, D, page = 2, 5, 2, 64, 16
    fused = torch.from_numpy(rng.standard_normal((B, T, 3 * H, D)).astype(np.float32)).to(dev())
    k, v = fused[:, :, H:2 * H], fused[:, :, 2 * H:]
    table = torch.tensor([[1], [0]], dtype=torch.int32, device=dev())
    st = torch.tensor([2, 9], dtype=torch.int32, device=dev())
    caches = [fgq.kv_cache(2, page, H, D, 32) for _ in range(2)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    fgq.fgq_kv_append(caches[0], k, v, table, st, stream=side)
    side.synchronize()
    fgq.fgq_kv_append(caches[1], k.contiguous(), v.contiguous(), table, st)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    for n in ("k_codes", "k_params", "v_codes", "v_params"):
        assert torch.equal(getattr(caches[0], n), getattr(caches[1], n)) and getattr(caches[0], n).any()


def test_nonfinite_groups_and_bad_pages():
    B, T, H, D, G, page = 1, 18, 1, 64, 32, 16
    x = torch.randn((B, T, H, D), device=dev())
    x[0, 2, 0, 5] = float("nan")
    x[0, 3, 0, 40] = float("inf")
    cache = fgq.kv_cache(2, page, H, D, G)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=dev())
    zero = torch.zeros(1, dtype=torch.int32, device=dev())
    fgq.fgq_kv_append(cache, x, x, table, zero)
    assert fgq.fgq_stream_status() == fgq.FGQ_ERR_NONFINITE
    k, _ = fgq.fgq_kv_read(cache, table, zero, T, dtype=torch.float32)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    assert not k[0, 2, 0, :32].any() and k[0, 2, 0, 32:].any()
    assert not k[0, 3, 0, 32:].any() and k[0, 3, 0, :32].any()
    # a page outside the pool, an unused entry, a position past the table, a negative start: reported, not touched
    before = cache.k_codes.clone()
    ok = torch.randn((B, T, H, D), device=dev())
    for bad, start in (([[1, 2]], 0), ([[1, -1]], 0), ([[1]], 0), ([[1, 0]], -3)):
        t = torch.tensor(bad, dtype=torch.int32, device=dev())
        s = torch.tensor([start], dtype=torch.int32, device=dev())
        fgq.fgq_kv_append(cache, ok, ok, t, s)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_ARG
        assert torch.equal(cache.k_codes[0], before[0])
        fgq.fgq_kv_read(cache, t, s, T)
        assert fgq.fgq_stream_status() == fgq.FGQ_ERR_ARG


def test_huge_and_tiny_values():
    """Groups whose range passes fp32's largest value, and subnormal ones, stay finite and within half a step."""
    D, G = 64, 32
    x = torch.zeros((1, 3, 1, D))
    x[0, 0, 0, :32] = torch.linspace(-3.3e38, 3.3e38, 32, dtype=torch.float64).float()  # fp32 steps would overflow
    x[0, 0, 0, 32:] = torch.linspace(3.0e38, 3.39e38, 32)
    x[0, 1, 0] = torch.linspace(-1e-39, 1e-39, 64)
    x[0, 2, 0] = torch.linspace(1e20, 1.01e20, 64)
    cache = fgq.kv_cache(1, 16, 1, D, G)
    table = torch.zeros((1, 1), dtype=torch.int32, device=dev())
    zero = torch.zeros(1, dtype=torch.int32, device=dev())
    fgq.fgq_kv_append(cache, x.to(dev()), x.to(dev()), table, zero)
    k, v = fgq.fgq_kv_read(cache, table, zero, 3, dtype=torch.float32)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    p = cache.k_params[0, 0, :3].cpu().numpy().view(np.uint32)
    lo, s = (p & 0xFFFF0000).view(np.float32).astype(np.float64), (p << np.uint32(16)).view(np.float32).astype(np.float64)
    c = R.unpack_codes(cache.k_codes[0, 0, :3].cpu().numpy(), True).astype(np.float64)
    back = np.repeat(lo, G, -1) + np.repeat(s, G, -1) * c
    assert np.all(np.isfinite(back)) and torch.equal(k, v)
    err = np.abs(back - x[0, :, 0].double().numpy())
    assert np.all(err <= np.repeat(s, G, -1) * 0.50001)


def test_long_cache_offsets():
    """Rows beyond 2^32 bytes of codes."""
    H, D, G, page = 8, 128, 128, 4096
    pages = 2200  # 2200 * 8 * 4096 * 64 bytes = 4.6 GB of key codes
    shape = (pages, H, page, D // 2)
    cache = fgq.KVCache(torch.empty(shape, dtype=torch.uint8, device=dev()),
                        torch.empty(shape[:3] + (1,), dtype=torch.int32, device=dev()),
                        torch.empty(shape, dtype=torch.uint8, device=dev()),
                        torch.empty(shape[:3] + (1,), dtype=torch.int32, device=dev()))
    x = torch.randn((1, 40, H, D), device=dev(), dtype=torch.bfloat16)
    y = torch.randn((1, 40, H, D), device=dev(), dtype=torch.bfloat16)
    table = torch.tensor([[pages - 1, 1]], dtype=torch.int32, device=dev())
    start = torch.tensor([page - 20], dtype=torch.int32, device=dev())
    fgq.fgq_kv_append(cache, x, y, table, start)
    k, v = fgq.fgq_kv_read(cache, table, start, 40, dtype=torch.float32)
    q = torch.randn((1, 1, H, D), device=dev(), dtype=torch.bfloat16)
    n = torch.tensor([page + 20], dtype=torch.int32, device=dev())
    o = fgq.fgq_kv_attention(q, cache, table, n, window=40)
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
    for got, want in ((k, x), (v, y)):
        w = want.float().cpu().numpy()
        c, lo, s = R.quantize4(w, G)
        assert np.array_equal(got.cpu().numpy(), R.dequantize4(c, lo, s).astype(np.float32))
    z = torch.einsum("hd,thd->ht", q[0, 0].double(), k[0].double()) * D ** -0.5
    want = torch.einsum("ht,thd->hd", torch.softmax(z, -1), v[0].double())
    assert (o[0, 0].double() - want).abs().max().item() <= 2 ** -8 * 4 + 2 ** -11 * 8


def test_empty_calls():
    cache = fgq.kv_cache(1, 16, 2, 64, 64)
    table = torch.zeros((1, 1), dtype=torch.int32, device=dev())
    zero = torch.zeros(1, dtype=torch.int32, device=dev())
    launches = fgq.fgq_launch_count()
    x = torch.empty((1, 0, 2, 64), device=dev())
    fgq.fgq_kv_append(cache, x, x, table, zero)
    k, _ = fgq.fgq_kv_read(cache, table, zero, 0)
    assert k.shape == (1, 0, 2, 64) and fgq.fgq_launch_count() == launches
    # lens of zero write nothing and read zeros
    x = torch.randn((1, 3, 2, 64), device=dev())
    fgq.fgq_kv_append(cache, x, x, table, zero, lens=zero)
    k, v = fgq.fgq_kv_read(cache, table, zero, 3, lens=zero)
    assert not cache.k_codes.any() and not k.any() and not v.any()
    assert fgq.fgq_stream_status() == fgq.FGQ_OK
