"""A small language model of attention layers, for running the decoder with a key-value cache.

Pre-norm layers of grouped-query attention and a two-layer perceptron, learned-looking random weights in
bf16, sinusoidal positions, tied to nothing.  It is an input producer like StandInLM: dense products are torch's stock
matmul; attention and cache are the package's operators.
"""
from __future__ import annotations

import math

import torch

import paper_2504_09135_b200 as disc


class AttentionLM:
    """V tokens, `layers` layers, width hq * d, hq query heads over hkv key heads of d values."""

    def __init__(self, V: int, layers: int, hq: int, hkv: int, d: int, *, seed: int = 0, device="cuda"):
        self.V, self.layers, self.hq, self.hkv, self.d, self.width = V, layers, hq, hkv, d, hq * d
        self.device = torch.device(device)
        gen = torch.Generator(device=self.device).manual_seed(seed)

        def weight(rows, cols, scale=None):
            w = torch.randn((rows, cols), generator=gen, device=self.device) * (scale or 1.0 / math.sqrt(rows))
            return w.to(torch.bfloat16)

        w = self.width
        self.embed = weight(V, w, 1.0)
        self.blocks = [dict(qkv=weight(w, (hq + 2 * hkv) * d), out=weight(w, w), up=weight(w, 2 * w), down=weight(2 * w, w))
                       for _ in range(layers)]
        self.head = weight(w, V)

    @staticmethod
    def norm(x: torch.Tensor) -> torch.Tensor:
        x32 = x.float()
        return (x32 * torch.rsqrt(x32.square().mean(dim=-1, keepdim=True) + 1e-6)).to(x.dtype)

    def positions(self, pos: torch.Tensor) -> torch.Tensor:
        f = torch.exp(torch.arange(0, self.width, 2, device=self.device) * (-math.log(10000.0) / self.width))
        a = pos.float()[:, None] * f[None, :]
        return torch.cat([torch.sin(a), torch.cos(a)], dim=1).to(torch.bfloat16)

    def run(self, tokens: torch.Tensor, pos: torch.Tensor, attend) -> torch.Tensor:
        """Final hidden vectors of the tokens; attend(layer, q, k, v) gives the attention's output [n, hq, d]."""
        x = self.embed.index_select(0, tokens.long()) + self.positions(pos)
        for i, b in enumerate(self.blocks):
            qkv = (self.norm(x) @ b["qkv"]).view(-1, self.hq + 2 * self.hkv, self.d)
            q, k, v = qkv.split([self.hq, self.hkv, self.hkv], dim=1)
            x = x + attend(i, q, k, v).reshape(-1, self.width) @ b["out"]
            x = x + torch.nn.functional.silu(self.norm(x) @ b["up"]) @ b["down"]
        return self.norm(x)

    def logits(self, hidden: torch.Tensor) -> torch.Tensor:
        return hidden @ self.head

    # ---- with the package's attention and cache -----------------------------------------------------------
    def new_cache(self, n_rows: int, longest: int, *, n_pages: int, page_size: int = 16) -> "disc.DiscCache":
        return disc.DiscCache.empty(self.layers, n_pages, page_size, self.hkv, self.d, n_rows, -(-longest // page_size) + 1,
                                    device=self.device)

    @torch.no_grad()
    def prefill(self, tokens: torch.Tensor, cu: torch.Tensor, max_len: int, cache=None, rows: torch.Tensor | None = None,
                status=None) -> torch.Tensor:
        """All tokens of packed sequences (cu int32[n + 1] on the device) -> hidden vectors [n tokens, width].  With a cache the keys
        and values go to its rows `rows`, which have been extended by the sequences' lengths."""
        at = torch.arange(tokens.numel(), device=self.device)
        seq = torch.searchsorted(cu.long(), at, right=True) - 1

        def attend(layer, q, k, v):
            if cache is not None:
                disc.disc_cache_write(cache, layer, k, v, cu=cu, rows=rows, status=status)
            return disc.disc_attend_prompt(q, k, v, cu, max_len=max_len)[0]

        return self.run(tokens, at - cu.long()[seq], attend)

    @torch.no_grad()
    def step(self, tokens: torch.Tensor, cache, plan, status=None) -> torch.Tensor:
        """One new token in every row of the cache, which has been extended by it -> hidden vectors [rows, width]."""

        def attend(layer, q, k, v):
            disc.disc_cache_write(cache, layer, k, v, status=status)
            return disc.disc_attend_cached(cache, layer, q, plan)[0]

        return self.run(tokens, (cache.len - 1).clamp(min=0), attend)

    @torch.no_grad()
    def score(self, tokens: torch.Tensor, cu: torch.Tensor, max_len: int, *, top: int = 0):
        """log P of every token after the first of each packed sequence, given those before it -> what disc_logprobs gives for the
        n tokens (the last token of a sequence has no next one: target -1)."""
        hidden = self.prefill(tokens, cu, max_len)
        nxt = torch.cat([tokens[1:], tokens.new_full((1,), -1)]).to(torch.int32)
        nxt[cu[1:].long() - 1] = -1
        return disc.disc_logprobs(self.logits(hidden), nxt, top=top)
