"""One attention block of a decoder, served from quantized state: the operators of include/fgq_decoder.h together.

Queries, keys and values come from one linear layer on 8-bit integers (a scale per token and per output channel), keys and
values go into a paged cache held in 4 bits, attention reads that cache, and a second 8-bit layer projects its output:

    qkv  = fgq_linear_w8a8(x)                 one call; q, k, v are views of its output
    cache[starts + i] = 4 bits of k, v        fgq_kv_append
    o    = softmax(q k^T / sqrt(D)) v         fgq_kv_attention, over everything cached so far
    y    = fgq_linear_w8a8(o)

The same call serves a prompt, a chunk of one, a few drafted tokens, and single tokens; sequences of a batch may
have different lengths.  (Position rotation, norms and the feed-forward part of a decoder layer are not here.)

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
                 window: int = 0):
        if q_heads % kv_heads:
            raise ValueError("kv_heads must divide q_heads")
        if wqkv.shape[0] != (q_heads + 2 * kv_heads) * head_dim or wo.shape != (wqkv.shape[1], q_heads * head_dim):
            raise ValueError("wqkv is [(q_heads + 2 kv_heads) head_dim][width], wo [width][q_heads head_dim]")
        self.q_heads, self.kv_heads, self.head_dim, self.window = q_heads, kv_heads, head_dim, window
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
        q, k, v = qkv.view(B, T, sum(heads), self.head_dim).split(heads, dim=2)
        fgq.fgq_kv_append(self.cache, k, v, self.pool.table, starts_d, lens=lens_d)
        o = fgq.fgq_kv_attention(q, self.cache, self.pool.table, ends_d, q_lens=lens_d, window=self.window,
                                 max_len=max(ends))
        self.pool.lengths = ends
        return fgq.fgq_linear_w8a8(o.view(B * T, self.q_heads * self.head_dim), *self.wo).view(B, T, width)


def main() -> None:
    torch.manual_seed(0)
    width, q_heads, kv_heads, D, B, T = 1024, 8, 2, 128, 2, 300
    w = torch.randn(((q_heads + 2 * kv_heads) * D, width), device="cuda") / width ** 0.5
    wo = torch.randn((width, q_heads * D), device="cuda") / (q_heads * D) ** 0.5
    block = AttentionBlock(w, wo, q_heads, kv_heads, D, pages=16, sequences=B)
    x = torch.randn((B, T + 8, width), device="cuda").to(torch.bfloat16)
    y = [block.forward(x[:, :T], lens=[T, T - 45])]          # two prompts of different lengths
    y += [block.forward(x[:, T + i:T + i + 1]) for i in range(8)]  # eight tokens each
    status = fgq.fgq_stream_status()
    c = block.cache
    held = sum(t.numel() * t.element_size() for t in (c.k_codes, c.k_params, c.v_codes, c.v_params))
    print(f"lengths {block.lengths}, last output rms {y[-1].float().square().mean().sqrt().item():.4f}, status {status}, "
          f"cache of {c.pages} pages {held / 1e6:.2f} MB ({2 * 2 * c.pages * c.page_size * kv_heads * D / 1e6:.2f} in bf16)")


if __name__ == "__main__":
    main()
