"""The decoder block (decoder.py): its operators together, against their definitions chained in 64 bits."""
import numpy as np
import pytest
import torch

import _decoder as R
from _gpu import dev
from paper_1705_01462_gb300 import decoder, fgq

pytestmark = pytest.mark.gpu


def block(seed, width, q_heads, kv_heads, D, G, page, pages, B, window=0):
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    w = torch.randn(((q_heads + 2 * kv_heads) * D, width), generator=g, device=dev()) / width ** 0.5
    wo = torch.randn((width, q_heads * D), generator=g, device=dev()) / (q_heads * D) ** 0.5
    return decoder.AttentionBlock(w, wo, q_heads, kv_heads, D, pages=pages, page_size=page, group=G, sequences=B,
                                  window=window), g


def defined(b, x, q_heads, kv_heads, D, G, window=0):
    """fp32 block output for whole sequences x [n][width] given one by one, 64 bits between the roundings that the
    operators define (8-bit tokens, 4-bit keys and values); the attention output's fp32 rounding is left out."""
    wq, ws = (t.cpu().numpy() for t in b.wqkv)
    woq, wos = (t.cpu().numpy() for t in b.wo)
    q8, s8 = R.quantize8(x)
    qkv, _ = R.linear(q8, s8, wq, ws, None, "f32")
    qkv = qkv.astype(np.float32).reshape(x.shape[0], -1, D)
    q, k, v = qkv[:, :q_heads], qkv[:, q_heads:q_heads + kv_heads], qkv[:, q_heads + kv_heads:]
    kd, vd = (R.dequantize4(*R.quantize4(t, G)) for t in (k, v))
    n, group = x.shape[0], q_heads // kv_heads
    o = np.zeros((n, q_heads, D))
    for i in range(n):
        lo = max(0, i + 1 - window) if window else 0
        for h in range(q_heads):
            z = kd[lo:i + 1, h // group] @ q[i, h].astype(np.float64) * D ** -0.5
            p = np.exp(z - z.max())
            o[i, h] = p @ vd[lo:i + 1, h // group] / p.sum()
    oq, os_ = R.quantize8(o.reshape(n, -1).astype(np.float32))
    return R.linear(oq, os_, woq, wos, None, "f32")[0], os_


@pytest.mark.parametrize("window", [0, 20])
def test_prompt_then_tokens(window):
    """A ragged prompt and single tokens, fp32.  The second layer quantizes the attention output, whose rounding
    (1e-5 of it at most) may move a code by one: half a step of every code is the tolerance, far above what it takes
    and far below a wrong key, value or position."""
    width, Hq, Hkv, D, G, B = 96, 4, 2, 64, 32, 2
    b, g = block(3, width, Hq, Hkv, D, G, 16, 12, B, window)
    x = torch.randn((B, 60, width), generator=g, device=dev())
    lens = [50, 33]
    got = [[], []]
    y = b.forward(x[:, :50], lens=lens)
    for s in range(B):
        got[s].append(y[s, :lens[s]])
    for i in range(6):
        y = b.forward(torch.stack([x[s, lens[s] + i] for s in range(B)])[:, None])
        for s in range(B):
            got[s].append(y[s])
    assert fgq.fgq_stream_status() == fgq.FGQ_OK and b.lengths == [56, 39]
    woq, wos = (t.cpu().numpy().astype(np.float64) for t in b.wo)
    for s in range(B):
        n = lens[s] + 6
        want, step = defined(b, x[s, :n].cpu().numpy(), Hq, Hkv, D, G, window)
        bound = 0.5 * step[:, None] * np.abs(woq * wos[:, None]).max(1) * 8 + 1e-4
        R.check(torch.cat(got[s]).cpu().numpy(), want, bound, "block")


def test_pieces_of_a_prompt():
    """A prompt in one call, in chunks, or token by token fills the cache with the same bytes (sums of the products
    are exact, whichever kernel forms them), and gives nearly the same outputs."""
    width, Hq, Hkv, D, G = 128, 8, 2, 128, 64
    x = torch.randn((1, 96, width), device=dev()).to(torch.bfloat16)
    outs, caches = [], []
    for cuts in ([96], [40, 41, 15], [1] * 96):
        b, _ = block(5, width, Hq, Hkv, D, G, 16, 8, 1)
        at, y = 0, []
        for c in cuts:
            y.append(b.forward(x[:, at:at + c]))
            at += c
        assert fgq.fgq_stream_status() == fgq.FGQ_OK
        outs.append(torch.cat(y, 1).float())
        c = b.cache
        caches.append([t.clone() for t in (c.k_codes, c.k_params, c.v_codes, c.v_params)])
    for c in caches[1:]:
        assert all(torch.equal(u, v) for u, v in zip(c, caches[0]))
    for o in outs[1:]:
        # bf16 attention outputs, 8-bit codes of them, bf16 outputs: a few roundings of 2^-8 and 1 / 127
        assert (o - outs[0]).abs().max().item() <= 0.05 * outs[0].abs().max().item()


def test_pool_and_refusals():
    pool = decoder.PagePool(3, 16, 2, 2, device=dev())
    pool.reserve([17, 16])
    assert sorted(pool.table.flatten().tolist()) == [-1, 0, 1, 2]
    with pytest.raises(RuntimeError):
        pool.reserve([17, 17])
    pool.release(0)
    pool.reserve([0, 30])
    assert pool.table[0].tolist() == [-1, -1] and -1 not in pool.table[1].tolist()
    with pytest.raises(ValueError):
        block(1, 64, 3, 2, 64, 32, 16, 2, 1)
    b, _ = block(1, 64, 2, 1, 64, 32, 16, 2, 1)
    with pytest.raises(ValueError):
        b.forward(torch.zeros((2, 1, 64), device=dev()))
    with pytest.raises(ValueError):
        b.forward(torch.zeros((1, 2, 64), device=dev()), lens=[3])


def test_main():
    decoder.main()
