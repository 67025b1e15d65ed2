"""A paged key-value cache for serving: the pages of every layer, who owns them, and attention over them.

    cache = PagedCache(layers=2, requests=64, kv_heads=4, head_dim=128, page=16, n_pages=4096, max_tokens=8192)
    cache.step(new_lens, n_new)                  # once per model step: pages taken and given back, slots of the new tokens
    for layer in range(2):
        q, k = api.fb_rotary_fwd(q, k, cache.positions[None], freqs, sections)       # or ALiBi slopes, or factors
        cache.append(layer, k, v)
        out, lse = cache.attend(layer, q)

new_lens [requests] int32 holds the tokens that each request is to have after the step: one more than before in decode,
the prompt's length for a new one, 0 for one that has ended (its pages go back), fewer for drafted tokens that are not
kept.  Everything stays on the device: a step synchronises nothing, reads nothing back, and can be captured into a graph.
A request for which no pages are left keeps its length (lens == starts; its queries come out as 0, lse -inf).
"""
from __future__ import annotations

from typing import Optional

import torch

from . import api


class PagedCache:
    def __init__(self, layers: int, requests: int, kv_heads: int, head_dim: int, page: int, n_pages: int, max_tokens: int,
                 rank: int = 0, dtype=torch.bfloat16, phi_dtype=torch.float32, device="cuda"):
        """n_pages of `page` tokens in each layer; a request may hold up to max_tokens.  rank: factors of a low-rank bias
        cached beside the keys (0: none)."""
        if min(layers, requests, kv_heads, n_pages, max_tokens) < 1 or rank < 0:
            raise api.FlashBiasError("sizes must be positive")
        if page not in (16, 32, 64, 128, 256):
            raise api.FlashBiasError("page must be 16, 32, 64, 128 or 256")
        blocks = -(-max_tokens // page)
        if requests > 4096 or n_pages * page >= 1 << 31 or requests * blocks >= 1 << 31:
            raise api.FlashBiasError("at most 4096 requests, and fewer than 2^31 tokens and table entries")
        self.page = page
        shape = (layers, n_pages, kv_heads, page)
        self.k_pages = torch.empty((*shape, head_dim), dtype=dtype, device=device)
        self.v_pages = torch.empty((*shape, head_dim), dtype=dtype, device=device)
        self.phi_pages = torch.empty((*shape, rank), dtype=phi_dtype, device=device) if rank else None
        self.table = torch.full((requests, blocks), -1, dtype=torch.int32, device=device)
        self.ring = torch.arange(n_pages, dtype=torch.int32, device=device)
        # lengths and the ring's (head, count), now and before the step
        self._now = torch.zeros(requests + 2, dtype=torch.int32, device=device)
        self._now[requests + 1] = n_pages
        self._before = self._now.clone()
        self.lens, self.starts = self._now[:requests], self._before[:requests]
        self.slots: Optional[torch.Tensor] = None
        self.positions: Optional[torch.Tensor] = None

    def step(self, new_lens: torch.Tensor, n_new: int) -> None:
        """From lens to new_lens, at most n_new new tokens a request: sets starts (the lengths before), lens, slots and
        positions [requests, n_new].  A step that is refused (it raises) leaves everything as it was."""
        b = self.table.shape[0]
        if not 1 <= n_new < (1 << 31) // b:
            raise api.FlashBiasError("n_new must be at least 1, and requests * n_new below 2^31")
        args, out = api._plan_call(self.starts, new_lens, self.table, self.ring, self._before[b:], n_new, self.page, self.lens,
                                   self._now[b:])
        self._before.copy_(self._now)
        api._run_plan(args)
        _, _, self.slots, self.positions = out

    def _layer_factors(self, layer: int):
        return None if self.phi_pages is None else self.phi_pages[layer]

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, phi_k: Optional[torch.Tensor] = None) -> None:
        """Stores the step's keys and values [requests, kv_heads, n_new, head_dim] (and factors) of one layer."""
        if self.slots is None:
            raise api.FlashBiasError("append needs a step before it")
        api.fb_paged_append(k, v, self.slots, self.k_pages[layer], self.v_pages[layer], phi_k, self._layer_factors(layer))

    def attend(self, layer: int, q: torch.Tensor, phi_q: Optional[torch.Tensor] = None, slopes: Optional[torch.Tensor] = None,
               scale: float = 0.0, causal: bool = True):
        """out, lse of the step's queries [requests, heads, n_new, head_dim] over everything their requests hold."""
        return api.fb_paged_attn_fwd(q, self.k_pages[layer], self.v_pages[layer], self.table, self.lens, self.starts, phi_q,
                                     self._layer_factors(layer), slopes, causal=causal, scale=scale)
