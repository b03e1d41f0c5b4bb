"""The verifier's keys and values between steps, over the C ABI.

A PagedCache owns the pool of 8-bit pages of every layer, the block table, the sequences' lengths and the stack of
free pages, all allocated once with torch on the target device. A speculative step uses it as

    attend (every layer)  ->  tf_sample  ->  tf_accept_walk  ->  grow  ->  append (every layer)

`attend` sees the tokens cached before the step and the drafted nodes' own keys and values; `grow` makes room for the
accepted path and `append` quantises it into its pages. Nothing here synchronises; `status` does.

A sequence that `grow` refuses keeps its length and has no slots, while its new tokens may already be drawn: who goes on
with it has to look at plan_status (the last change's words) or at `status`, which keeps every refusal.

Everything that a call does - its kernels, and the tensors that it makes where none are passed - happens on the stream
that it is given (none: the current one), so a tensor that it returns belongs to that stream. Calls of one cache have
to be ordered among each other, as calls on one stream are: they share the lengths, the pages and one workspace.
"""
from __future__ import annotations

import math
from contextlib import nullcontext

import torch

from . import binding as B


def _on(stream):
    return nullcontext() if stream is None else torch.cuda.stream(stream)


class PagedCache:
    def __init__(self, dims: B.CacheDims, layers: int = 1, n_max: int = 1, device="cuda"):
        """layers: caches that share the block table; n_max: most new tokens per sequence of one `attend`."""
        B.load_library()
        self.dims, self.layers = dims, layers
        dev = torch.device(device)
        i32 = dict(dtype=torch.int32, device=dev)
        pages = (layers, dims.n_pages, dims.kv_heads, dims.page, dims.head_dim)
        self.k = torch.zeros(pages, dtype=torch.uint8, device=dev)
        self.v = torch.zeros(pages, dtype=torch.uint8, device=dev)
        self.k_scale = torch.ones(pages[:3], dtype=torch.float32, device=dev)
        self.v_scale = torch.ones(pages[:3], dtype=torch.float32, device=dev)
        self.block_table = torch.full((dims.batch, dims.max_pages), -1, **i32)
        self.seq_len = torch.zeros(dims.batch, **i32)
        self.free_list = torch.arange(dims.n_pages - 1, -1, -1, **i32)
        self.free_count = torch.full((1,), dims.n_pages, **i32)
        self.plan_status = torch.zeros(dims.batch, **i32)
        self.dev_status = torch.zeros(dims.batch, **i32)
        self.ws = B.alloc_attention_workspace(dims, n_max, dev)

    def grow(self, delta, extra: int = 0, width: int = 0, slot_map=None, stream=None):
        """Change the lengths by delta + extra (delta = accept_len and extra = 1 for an accepted path) and return the
        new tokens' slots [batch, width]; a sequence that cannot grow keeps its length and has none: plan_status says why until
        the next change, `status` until `clear_status`."""
        if slot_map is None and width > 0:
            with _on(stream):
                slot_map = torch.empty((self.dims.batch, width), dtype=torch.int32, device=self.seq_len.device)
        B.tf_cache_plan(self.dims, self.seq_len, delta, extra, self.block_table, self.free_list, self.free_count, slot_map,
                        self.seq_len, self.plan_status, stream)
        with _on(stream):
            self.dev_status.bitwise_or_(self.plan_status)     # the next change overwrites plan_status
        return slot_map

    def release(self, which, stream=None):
        """Empty the sequences where `which` [batch] is true: their pages return to the pool."""
        with _on(stream):
            self.grow(torch.where(which, -self.seq_len, 0), stream=stream)

    def append(self, layer: int, k, v, slot_map, src=None, stream=None):
        B.tf_cache_append(self.dims, k, v, slot_map, src, self.k[layer], self.v[layer], self.k_scale[layer],
                          self.v_scale[layer], self.dev_status, stream)

    def attend(self, layer: int, q, k, v, mask=None, scale=None, out=None, lse=None, stream=None):
        """Attention of the new tokens over the cache and over themselves; returns out [batch, n, heads, head_dim]."""
        if out is None:
            with _on(stream):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        B.tf_tree_attention(self.dims, q, k, v, self.k[layer], self.v[layer], self.k_scale[layer], self.v_scale[layer],
                            self.block_table, self.seq_len, mask, scale if scale is not None else 1 / math.sqrt(self.dims.head_dim),
                            out, lse, self.dev_status, self.ws, stream)
        return out

    def status(self, stream=None) -> int:
        """Synchronise and return the TF_DEV_* flags of every call since the cache was made or `clear_status` was called; those
        of a single sequence are in dev_status."""
        flags = 0
        with _on(stream):
            for word in torch.cat([self.plan_status, self.dev_status]).tolist():
                flags |= word
        return flags

    def clear_status(self, stream=None):
        with _on(stream):
            self.plan_status.zero_()
            self.dev_status.zero_()
