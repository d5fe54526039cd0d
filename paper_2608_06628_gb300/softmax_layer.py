"""The attention of one softmax layer of a hybrid model: norm and rotation of queries and
keys with the cache write in one pass, then attention over the paged cache.

A layer works on the output of its fused projection, qkv [tokens, (Hq + 2 Hkv) d], and on a
PagePool whose append() has made room for those tokens.
"""
from __future__ import annotations

import torch

from . import hybrid as H
from .page_pool import OnStream, PagePool


class SoftmaxLayer:
    def __init__(self, cfg: H.hybrid_cfg, rope, wq=None, wk=None, window: int = 0, n_sink: int = 0):
        """rope: what hybrid.make_rope returns; wq, wk: norm weights [d] in the io type, or None."""
        self.cfg, (self.rope, self.freqs) = cfg, rope
        self.wq, self.wk, self.window, self.n_sink = wq, wk, window, n_sink

    def split(self, qkv):
        """Q, K, V as views [tokens, heads, d] of the projection's output."""
        c = self.cfg
        q, k, v = qkv.split([c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim, c.n_kv_heads * c.head_dim], dim=-1)
        return (x.unflatten(-1, (-1, c.head_dim)) for x in (q, k, v))

    def write(self, qkv, pool: PagePool, layer: int, slots, positions, stream=None):
        """Normalise and rotate; keys and values go to their slots.  Returns the queries."""
        q, k, v = self.split(qkv)
        kc, vc = pool.k_cache[layer], pool.v_cache[layer]
        with OnStream(stream, qkv, slots, positions, self.wq, self.wk, self.freqs, kc, vc) as on:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            H.hybrid_qk_norm_rope_cache(self.cfg, self.rope, pool.pg, q, q.stride(0), k, k.stride(0), v, v.stride(0), q.shape[0],
                                        self.wq, self.wk, positions, self.freqs, slots, out, kc, vc)
            return on.returns(out)

    def attend(self, q, pool: PagePool, layer: int, stream=None):
        """q [n_req * B, Hq, d] of the active blocks against the cache -> the same shape."""
        kc, vc = pool.k_cache[layer], pool.v_cache[layer]
        with OnStream(stream, q, kc, vc, pool.block_table, pool.lens) as on:
            out, workspace = torch.empty_like(q), pool.workspace_of(self.cfg, on)
            H.hybrid_paged_attn(self.cfg, pool.pg, q, kc, vc, pool.block_table, pool.lens, pool.n_req, self.window, self.n_sink,
                                out, workspace, workspace.numel())
            return on.returns(out)

    def step(self, qkv, pool: PagePool, layer: int, slots, positions, stream=None):
        """One denoising step of the active blocks (or, with B = 1, one token)."""
        return self.attend(self.write(qkv, pool, layer, slots, positions, stream), pool, layer, stream)
