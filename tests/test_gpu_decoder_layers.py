"""Whole decoder layers (decoder.Decoder): the operators together, against their definitions chained in 64 bits."""
import numpy as np
import pytest
import torch

import _decoder as D8
import _layer as R
from _gpu import dev
from paper_1705_01462_gb300 import decoder, fgq

pytestmark = pytest.mark.gpu

WIDTH, HQ, HKV, D, G, HIDDEN, EXPERTS, TOP, OUT, FACTOR = 96, 4, 2, 64, 32, 80, 6, 2, 50, 4.0


def model(seed, B, mixed):
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device=dev()) / s[-1] ** 0.5  # noqa: E731
    norm = lambda: fgq.Norm(1 + 0.2 * torch.randn(WIDTH, generator=g, device=dev()), eps=1e-5)  # noqa: E731
    table = fgq.rope_table(D, scaling="ramp", factor=FACTOR, length=40.0, high=4.0, device=dev())
    a = decoder.AttentionBlock(rnd((HQ + 2 * HKV) * D, WIDTH), rnd(WIDTH, HQ * D), HQ, HKV, D, pages=12, page_size=16, group=G,
                               sequences=B, rope=table, rope_layout="interleaved")
    if mixed:
        f = decoder.FeedForward(rnd(EXPERTS, HIDDEN, WIDTH), rnd(EXPERTS, HIDDEN, WIDTH), rnd(EXPERTS, WIDTH, HIDDEN),
                                router=rnd(EXPERTS, WIDTH), top=TOP, group=G, scale=1.5)
    else:
        f = decoder.FeedForward(rnd(HIDDEN, WIDTH), rnd(HIDDEN, WIDTH), rnd(WIDTH, HIDDEN), group=G)
    m = decoder.Decoder([(norm(), a, norm(), f)], norm(), rnd(OUT, WIDTH), posts=[(norm(), None)], scale=0.5, group=G)
    return m, g


def rms(z, n):
    return z / np.sqrt((z * z).mean(-1, keepdims=True) + n.eps) * n.weight.double().cpu().numpy()


def defined(m, x, mixed, out8):
    """Outputs for the tokens x fp64 [n][WIDTH] of one sequence.  The 8-bit and 4-bit roundings of a chain are decisions that fp32
    roundings can turn, so the attention block's output is taken from the device (out8); its own chain has tests of its own."""
    (n0, _, n1, f), (post, _) = m.layers[0], m.posts[0]
    s = x + 0.5 * rms(out8, post)
    y = rms(s, n1)
    w = [fgq.fgq_read_weights_w4(v).double().cpu().numpy().reshape((-1, v.rows, v.cols)) for v in f.weights]
    if mixed:
        ids, g, _ = R.route(y, f.router.double().cpu().numpy(), TOP, "softmax", True, 1.5)
    else:
        ids, g = np.zeros((len(x), 1), int), np.ones((len(x), 1))
    z, _ = R.experts(y, ids, g, np.zeros((len(x), 1)), *w, G, G, "f32")
    y = rms(s + 0.5 * z, m.last)
    return y @ fgq.fgq_read_weights_w4(m.head).double().cpu().numpy().T


@pytest.mark.parametrize("mixed", [False, True])
def test_prompt_then_tokens(mixed):
    """fp32: a ragged prompt, then single tokens.  Three norms and three products in a row, each within 2^-17 of its terms'
    magnitudes (_layer.beta), and factors of at most 10 between an error and what the next operator makes of it: 1e-3 of the largest output, far
    below a wrong expert, position or norm.  No token's experts lie nearer one another than that."""
    B = 2
    m, g = model(3, B, mixed)
    block = m.layers[0][1]
    seen = [[], []]
    forward = block.forward
    x = torch.randn((B, 40, WIDTH), generator=g, device=dev())
    lens, got = [30, 17], [[], []]

    def watch(y, n=None):
        out = forward(y, n)
        for b in range(B):
            seen[b].append(out[b, :y.shape[1] if n is None else n[b]].clone())
        return out

    block.forward = watch
    y = m.forward(x[:, :30], lens=lens)
    for b in range(B):
        got[b].append(y[b, :lens[b]])
    for i in range(5):
        y = m.forward(torch.stack([x[b, lens[b] + i] for b in range(B)])[:, None])
        for b in range(B):
            got[b].append(y[b])
    assert fgq.fgq_stream_status() == fgq.FGQ_OK and block.lengths == [35, 22]
    for b in range(B):
        n = lens[b] + 5
        want = defined(m, x[b, :n].double().cpu().numpy(), mixed, torch.cat(seen[b]).double().cpu().numpy())
        d = np.abs(torch.cat(got[b]).double().cpu().numpy() - want).max()
        assert d <= 1e-3 * np.abs(want).max(), d


def test_rotation_of_the_block():
    """The block with a table: keys in the cache are the turned ones (to the 4 bits' half step), at every position."""
    m, g = model(5, 1, False)
    block = m.layers[0][1]
    x = torch.randn((1, 20, WIDTH), generator=g, device=dev())
    for cut in (slice(0, 12), slice(12, 13), slice(13, 20)):
        block.forward(x[:, cut])
    qkv = fgq.fgq_linear_w8a8(x[0], *block.wqkv).view(20, -1, D).double().cpu().numpy()
    f = R.freqs(D, scaling="ramp", factor=FACTOR, length=40.0, high=4.0)
    want, bound = R.rope(qkv[None, :, HQ:HQ + HKV], f, [0], None, "interleaved", 1.0, False, "f32")
    zero = torch.zeros(1, dtype=torch.int32, device=dev())
    k, v = fgq.fgq_kv_read(block.cache, block.pool.table, zero, 20, dtype=torch.float32)
    step = (want.reshape(20, HKV, -1, G).max(-1) - want.reshape(20, HKV, -1, G).min(-1)) / 15 * (1 + 2.0 ** -6) + 2.0 ** -7
    tol = 0.51 * np.repeat(step, G, -1).reshape(want.shape) + bound
    R.check(k.double().cpu().numpy(), want, tol, "keys")
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_types_and_pieces():
    """16-bit streams; a prompt in one call or token by token gives nearly the same (a few roundings of 2^-8 and 1 / 127)."""
    for dtype in (torch.bfloat16, torch.float16):
        outs = []
        for cuts in ([24], [10, 1, 13], [1] * 24):
            m, g = model(7, 1, True)
            x = torch.randn((1, 24, WIDTH), generator=g, device=dev()).to(dtype)
            at, y = 0, []
            for c in cuts:
                y.append(m.forward(x[:, at:at + c]))
                at += c
            outs.append(torch.cat(y, 1).float())
            assert y[0].dtype == dtype
        assert fgq.fgq_stream_status() == fgq.FGQ_OK
        for o in outs[1:]:
            # a token whose second and third expert are nearly equal may take the other: few of them
            far = (o - outs[0]).abs().amax(-1) > 0.1 * outs[0].abs().max()
            assert far.float().mean().item() <= 0.1


def test_operators_in_a_graph():
    """A step of the operators around the cache, captured and replayed on new tokens."""
    m, g = model(9, 1, True)
    (n0, a, n1, f), (post, _) = m.layers[0], m.posts[0]
    x = torch.randn((3, WIDTH), generator=g, device=dev()).to(torch.bfloat16)
    f.router = f.router.to(torch.bfloat16)
    starts = torch.tensor([5, 9, 1000], dtype=torch.int32, device=dev())

    def step():
        s, y = fgq.fgq_add_norm(x, None, n0)
        q = fgq.fgq_linear_w8a8(y, *a.wqkv).view(3, 1, -1, D)
        q = fgq.fgq_rope(q, a.rope, starts, layout="interleaved", out=q)
        o = fgq.fgq_linear_w8a8(q.view(3, -1)[:, :HQ * D], *a.wo)
        s, y = fgq.fgq_add_norm(o, s, n1, post=post, residual_out=s)
        s, y = fgq.fgq_add_norm(f.forward(y), s, m.last, residual_out=s)
        return fgq.fgq_linear_w4(y, m.head)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step()
    for k in range(3):
        x.copy_(torch.randn(x.shape, generator=g, device=dev()))
        starts.add_(k)
        graph.replay()
        got = y.clone()
        assert torch.equal(got, step())
    assert fgq.fgq_stream_status() == fgq.FGQ_OK


def test_refusals():
    z = torch.zeros((8, 16), device=dev())
    with pytest.raises(ValueError):
        decoder.FeedForward(z, z, z)
    with pytest.raises(ValueError):
        decoder.FeedForward(z, z, z.t().contiguous(), router=torch.zeros((2, 16), device=dev()))
    with pytest.raises(ValueError):
        decoder.Decoder([], fgq.Norm(), z)
    m, _ = model(1, 2, False)
    with pytest.raises(ValueError):
        m.forward(torch.zeros((1, 1, WIDTH), device=dev()))
    m.forward(torch.zeros((2, 3, WIDTH), device=dev()))
    m.release(1)
    assert m.layers[0][1].lengths == [3, 0]


def test_main():
    decoder.main()
