"""Caller-side state of a serving loop on the paged key/value cache.

Allocation and bookkeeping only (PyTorch owns the memory, the library's kernels do every step): the cache of every
layer, the requests' lengths and block tables, the free list, and the arrays that a step's calls pass to one
another.  All of it stays on the device; a step needs nothing back from it to be issued.
"""
from __future__ import annotations

import torch

from . import binding as B


class PagedCache:
    """Keys and values of ``layers`` layers in ``n_pages`` pages of ``page_size`` tokens, and the state of up to
    ``requests`` requests of up to ``max_len`` tokens each.  fp8: e4m3 with the given scales [layers, kv_heads]."""

    def __init__(self, ctx: B.Context, *, layers, requests, max_tokens, max_len, n_pages, page_size, kv_heads, head_dim,
                 k_scale=None, v_scale=None, device="cuda"):
        self.ctx, self.page_size, self.max_tokens = ctx, page_size, max_tokens
        fp8 = k_scale is not None
        X, dtype = (16, torch.float8_e4m3fn) if fp8 else (8, torch.bfloat16)
        self.k = torch.zeros((layers, n_pages, kv_heads, head_dim // X, page_size, X), dtype=dtype, device=device)
        self.v = torch.zeros((layers, n_pages, kv_heads, page_size // X, head_dim, X), dtype=dtype, device=device)
        self.scales = (k_scale, v_scale)
        self.caches = [B.make_kv_cache(self.k[i], self.v[i], k_scale[i] if fp8 else None, v_scale[i] if fp8 else None)
                       for i in range(layers)]
        ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=device)  # noqa: E731
        self.table = torch.full((requests, -(-max_len // page_size)), -1, dtype=torch.int32, device=device)
        self.free_list = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.free = torch.full((1,), n_pages, dtype=torch.int32, device=device)
        self.lens, self.drops = ints(requests), ints(requests)
        self.q_offsets, self.status = ints(requests + 1), ints(4)
        self.slots, self.positions = ints(max_tokens), ints(max_tokens)

    def plan(self, new_lens, T: int):
        """Pages and slots of a step's T tokens, new_lens int32 [requests] on the device (-1: the request has ended).  What the
        last verification left in ``drops`` is taken back first, once: an accepted step clears it.  ``status`` tells a refused
        step, which changes nothing."""
        self.ctx.dx_pages_plan_in_place(new_lens, self.lens, self.drops, self.free, self.free_list, self.table, self.page_size,
                                        self.q_offsets, self.slots[:T], self.positions[:T], self.status)

    def write(self, layer: int, k, v):
        """k, v bf16 [T, kv_heads, head_dim] of the planned tokens (rows at any stride)."""
        self.ctx.dx_kv_write(self.caches[layer], k, v, self.slots[:k.shape[0]])

    def attend(self, layer: int, q, out, max_q: int, scale: float, window: int = 0, lse=None):
        """q, out bf16 [T, q_heads, head_dim] of the planned tokens, whose keys have been written."""
        self.ctx.dx_paged_attention(self.caches[layer], q, self.q_offsets, self.lens, self.table, max_q, scale, window, out, lse)

    def verify(self, p, q, draft, offsets, max_n: int, u_accept, u_sample, tokens, accepted):
        """Accepts drafts of the step planned last (all arrays as for ``dx_draft_verify``); the next ``plan`` drops the others.  A
        refused step gets no tokens, and the drops that its plan has not taken back stay."""
        self.ctx.dx_draft_verify_planned(self.status, p, q, draft, offsets, max_n, u_accept, u_sample, tokens, accepted, self.drops)
