"""A decoder served from quantized state: the operators of include/fgq_decoder.h together.

AttentionBlock.  Queries, keys and values come from one linear layer on 8-bit integers (a scale per token and per output
channel), queries and keys are turned by their positions (where a table is given), keys and values go into a paged cache
held in 4 bits, attention reads that cache, and a second 8-bit layer projects its output:

    qkv  = fgq_linear_w8a8(x)                 one call; q, k, v are views of its output
    q, k turned in place                      fgq_rope
    cache[starts + i] = 4 bits of k, v        fgq_kv_append
    o    = softmax(q k^T / sqrt(D)) v         fgq_kv_attention, over everything cached so far
    y    = fgq_linear_w8a8(o)

FeedForward.  A gated feed-forward layer, or a mixture of them, on 4-bit weights: fgq_moe_w4 (fgq_experts_w4 without a router).

Decoder.  Blocks one after another on a residual stream s, each pair of neighbours joined by one fgq_add_norm, which adds what a
block gives and normalises for the next, and a 4-bit layer to the outputs at the end (fgq_linear_w4):

    y = norm(s);  s, y = fgq_add_norm(block(y), s, next norm);  ...;  logits = fgq_linear_w4(y)

The same calls serve a prompt, a chunk of one, a few drafted tokens, and single tokens; sequences of a batch may
have different lengths.

``python -m paper_1705_01462_gb300.decoder`` runs a prompt and some decoding steps on random weights.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from paper_1705_01462_gb300 import fgq


class PagePool:
    """Hands out the pages of a cache and keeps the page table and the lengths of its sequences (host side)."""

    def __init__(self, pages: int, page_size: int, sequences: int, max_pages: int, device="cuda"):
        self.page_size = page_size
        self._free = list(range(pages - 1, -1, -1))
        self._held: List[List[int]] = [[] for _ in range(sequences)]
        self.table = torch.full((sequences, max_pages), -1, dtype=torch.int32, device=device)
        self.lengths = [0] * sequences  # tokens of each sequence in the cache

    def reserve(self, lengths: Sequence[int]) -> None:
        """Pages for sequences of these lengths; those that they hold already stay."""
        for b, n in enumerate(lengths):
            held = self._held[b]
            want = -(-n // self.page_size) - len(held)
            if want <= 0:
                continue
            if want > len(self._free) or len(held) + want > self.table.shape[1]:
                raise RuntimeError(f"no page left for sequence {b} of {n} tokens")
            new = [self._free.pop() for _ in range(want)]
            self.table[b, len(held):len(held) + want] = torch.tensor(new, dtype=torch.int32)
            held += new

    def release(self, b: int) -> None:
        """Ends sequence b: its pages are free, and its place holds no tokens."""
        self._free += reversed(self._held[b])
        self._held[b] = []
        self.table[b] = -1
        self.lengths[b] = 0


class AttentionBlock:
    """The block above: wqkv fp32 [(q_heads + 2 kv_heads) head_dim][width], wo fp32 [width][q_heads head_dim]."""

    def __init__(self, wqkv: torch.Tensor, wo: torch.Tensor, q_heads: int, kv_heads: int, head_dim: int, pages: int,
                 page_size: int = 64, group: int = 64, sequences: int = 1, max_pages: Optional[int] = None,
                 window: int = 0, rope: Optional[torch.Tensor] = None, rope_layout: str = "half"):
        """rope: a table of fgq.rope_table, or None (no rotation)."""
        if q_heads % kv_heads:
            raise ValueError("kv_heads must divide q_heads")
        if wqkv.shape[0] != (q_heads + 2 * kv_heads) * head_dim or wo.shape != (wqkv.shape[1], q_heads * head_dim):
            raise ValueError("wqkv is [(q_heads + 2 kv_heads) head_dim][width], wo [width][q_heads head_dim]")
        self.q_heads, self.kv_heads, self.head_dim, self.window = q_heads, kv_heads, head_dim, window
        self.rope, self.rope_layout = rope, rope_layout
        self.wqkv = fgq.fgq_quantize_weights_w8(wqkv)  # int8 and a scale per output channel
        self.wo = fgq.fgq_quantize_weights_w8(wo)
        self.cache = fgq.kv_cache(pages, page_size, kv_heads, head_dim, group, device=wqkv.device)
        self.pool = PagePool(pages, page_size, sequences, max_pages or pages, device=wqkv.device)

    @property
    def lengths(self) -> List[int]:
        """Tokens of each sequence in the cache."""
        return self.pool.lengths

    @lengths.setter
    def lengths(self, lengths: Sequence[int]) -> None:
        self.pool.lengths = list(lengths)

    def release(self, b: int) -> None:
        """Ends sequence b; the next tokens given in its place start another."""
        self.pool.release(b)

    def forward(self, x: torch.Tensor, lens: Optional[Sequence[int]] = None) -> torch.Tensor:
        """x [sequences][T][width] -> the same shape and type; lens[b] <= T tokens of sequence b are real (None: T), the
        others finite and their outputs of no meaning."""
        B, T, width = x.shape
        lens = [T] * B if lens is None else list(lens)
        if B != len(self.lengths) or len(lens) != B or any(n < 0 or n > T for n in lens):
            raise ValueError("x is [sequences][T][width] with 0 <= lens[b] <= T")
        ends = [n + m for n, m in zip(self.lengths, lens)]
        self.pool.reserve(ends)
        starts_d, lens_d, ends_d = torch.tensor([self.lengths, lens, ends], dtype=torch.int32, device=x.device)
        qkv = fgq.fgq_linear_w8a8(x.reshape(B * T, width), *self.wqkv)
        heads = [self.q_heads, self.kv_heads, self.kv_heads]
        qkv = qkv.view(B, T, sum(heads), self.head_dim)
        if self.rope is not None:
            turned = qkv[:, :, :self.q_heads + self.kv_heads]
            fgq.fgq_rope(turned, self.rope, starts_d, lens=lens_d, layout=self.rope_layout, out=turned)
        q, k, v = qkv.split(heads, dim=2)
        fgq.fgq_kv_append(self.cache, k, v, self.pool.table, starts_d, lens=lens_d)
        o = fgq.fgq_kv_attention(q, self.cache, self.pool.table, ends_d, q_lens=lens_d, window=self.window,
                                 max_len=max(ends))
        self.pool.lengths = ends
        return fgq.fgq_linear_w8a8(o.view(B * T, self.q_heads * self.head_dim), *self.wo).view(B, T, width)


class FeedForward:
    """A gated feed-forward layer, sum_j g_j down_e (silu(gate_e x) * (up_e x)): gate, up fp32 [experts][hidden][width], down
    [experts][width][hidden], quantized to 4 bits here; router [experts][width] (of the tokens' type or fp32) picks `top` experts a
    token.  Without a router: one layer, weights without the experts' axis."""

    def __init__(self, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor, router: Optional[torch.Tensor] = None,
                 top: int = 1, group: int = 64, score: str = "softmax", renormalize: bool = True, scale: float = 1.0):
        experts = 1 if router is None else router.shape[0]
        want = () if router is None else (experts,)
        hidden, width = gate.shape[-2:]
        if gate.shape != want + (hidden, width) or up.shape != gate.shape or down.shape != want + (width, hidden):
            raise ValueError("gate and up are [experts][hidden][width], down [experts][width][hidden]")
        self.weights = [fgq.fgq_quantize_weights_w4(w, group) for w in (gate, up, down)]
        self.router, self.top = router, top
        self.how = {"score": score, "renormalize": renormalize, "scale": scale}
        self.scale = scale

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x [tokens][width] -> the same shape and type."""
        if self.router is not None:
            return fgq.fgq_moe_w4(x, self.router, self.top, *self.weights, **self.how)
        ids = torch.zeros((x.shape[0], 1), dtype=torch.int32, device=x.device)
        return fgq.fgq_experts_w4(x, ids, torch.full(ids.shape, self.scale, device=x.device), *self.weights)


class Decoder:
    """Layers of an attention block and a feed-forward layer on a residual stream, a last norm, and a 4-bit layer to the outputs.

    layers: (norm, attention, norm, feed-forward), where a norm is what the block after it reads; posts: for each layer the norms of
    the two blocks' outputs, (Norm or None, Norm or None), or None; scale: what a block's output is multiplied by as it is
    added; head: fp32 [outputs][width]."""

    def __init__(self, layers, last: "fgq.Norm", head: torch.Tensor, posts=None, scale: float = 1.0, group: int = 64):
        if not layers or (posts is not None and len(posts) != len(layers)):
            raise ValueError("at least one layer, and posts for each or none")
        self.layers, self.last, self.scale = list(layers), last, scale
        self.posts = list(posts) if posts is not None else [(None, None)] * len(self.layers)
        self.head = fgq.fgq_quantize_weights_w4(head, group)

    def forward(self, x: torch.Tensor, lens: Optional[Sequence[int]] = None) -> torch.Tensor:
        """x [sequences][T][width], the residual stream's start -> outputs [sequences][T][outputs] of x's type; lens as
        AttentionBlock.forward.  x stays as it is."""
        B, T, width = x.shape
        s, y = fgq.fgq_add_norm(x.reshape(B * T, width), None, self.layers[0][0])
        for n, (_, attention, norm, feed) in enumerate(self.layers):
            after = self.layers[n + 1][0] if n + 1 < len(self.layers) else self.last
            o = attention.forward(y.view(B, T, width), lens).view(B * T, width)
            _, y = fgq.fgq_add_norm(o, s, norm, post=self.posts[n][0], scale=self.scale, residual_out=s, y=y)
            o = feed.forward(y)
            _, y = fgq.fgq_add_norm(o, s, after, post=self.posts[n][1], scale=self.scale, residual_out=s, y=y)
        return fgq.fgq_linear_w4(y, self.head).view(B, T, self.head.rows)

    def release(self, b: int) -> None:
        """Ends sequence b in every layer."""
        for _, attention, _, _ in self.layers:
            attention.release(b)


def main() -> None:
    torch.manual_seed(0)
    width, q_heads, kv_heads, D, B, T, hidden, experts, outputs = 1024, 8, 2, 128, 2, 300, 512, 8, 4096
    random = lambda *shape: torch.randn(shape, device="cuda") / shape[-1] ** 0.5  # noqa: E731
    norm = lambda: fgq.Norm(torch.ones(width, device="cuda"))  # noqa: E731
    table = fgq.rope_table(D, scaling="ramp", factor=4.0, length=4096.0)

    def attention():
        return AttentionBlock(random((q_heads + 2 * kv_heads) * D, width), random(width, q_heads * D), q_heads, kv_heads, D,
                              pages=16, sequences=B, rope=table)

    dense = FeedForward(random(hidden, width), random(hidden, width), random(width, hidden))
    mixed = FeedForward(random(experts, hidden, width), random(experts, hidden, width), random(experts, width, hidden),
                        router=random(experts, width).to(torch.bfloat16), top=2)
    model = Decoder([(norm(), attention(), norm(), dense), (norm(), attention(), norm(), mixed)], norm(), random(outputs, width))
    x = torch.randn((B, T + 8, width), device="cuda").to(torch.bfloat16)
    y = [model.forward(x[:, :T], lens=[T, T - 45])]          # two prompts of different lengths
    y += [model.forward(x[:, T + i:T + i + 1]) for i in range(8)]  # eight tokens each
    status = fgq.fgq_stream_status()
    block = model.layers[0][1]
    c = block.cache
    held = sum(t.numel() * t.element_size() for t in (c.k_codes, c.k_params, c.v_codes, c.v_params))
    print(f"lengths {block.lengths}, last outputs rms {y[-1].float().square().mean().sqrt().item():.4f}, status {status}, "
          f"cache of {c.pages} pages {held / 1e6:.2f} MB ({2 * 2 * c.pages * c.page_size * kv_heads * D / 1e6:.2f} in bf16)")


if __name__ == "__main__":
    main()
