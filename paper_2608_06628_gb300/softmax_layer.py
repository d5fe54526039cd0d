"""The attention of one softmax layer of a hybrid model: norm and rotation of queries and
keys with the cache write in one pass, then attention over the paged cache.

A layer works on the output of its fused projection, qkv [tokens, (Hq + 2 Hkv) d], and on a
PagePool whose append() has made room for those tokens. Shapes, types and layouts are checked
(ValueError) before anything is launched.

    slots, positions, offsets = pool.append(n_new, n_tok)
    rows = pool.block_rows(offsets, n_tok)     # unless every request has a whole block of new tokens
    out = layer.step(qkv, pool, i, slots, positions, rows=rows)
"""
from __future__ import annotations

import math

import torch

from . import hybrid as H
from .page_pool import BlockRows, OnStream, PagePool, expect


class SoftmaxLayer:
    def __init__(self, cfg: H.hybrid_cfg, rope, wq=None, wk=None, window: int = 0, n_sink: int = 0):
        """rope: what hybrid.make_rope returns; wq, wk: norm weights [d] in the io type, or None."""
        self.cfg, (self.rope, self.freqs) = cfg, rope
        self.wq, self.wk, self.window, self.n_sink = wq, wk, window, n_sink
        self.dtype = torch.bfloat16 if cfg.io_dtype == H.HYBRID_BF16 else torch.float32

    def _check_pool(self, pool: PagePool):
        """The caches are laid out by the pool's cfg and read by the layer's."""
        for name in ("head_dim", "n_kv_heads", "io_dtype"):
            if getattr(self.cfg, name) != getattr(pool.cfg, name):
                raise ValueError(f"pool: its caches are those of {pool.cfg}, the layer's of {self.cfg}")

    def split(self, qkv):
        """Q, K, V as views [tokens, heads, d] of the projection's output."""
        c = self.cfg
        q, k, v = qkv.split([c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim, c.n_kv_heads * c.head_dim], dim=-1)
        return (x.unflatten(-1, (-1, c.head_dim)) for x in (q, k, v))

    def write(self, qkv, pool: PagePool, layer: int, slots, positions, stream=None):
        """Normalise and rotate; keys and values go to their slots.  Returns the queries."""
        self._check_pool(pool)
        c, dev, n_tok = self.cfg, pool.device, qkv.shape[0]
        expect(qkv, "qkv", self.dtype, dev, n_tok, (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, rows=True)
        expect(slots, "slots", torch.int32, dev, max(n_tok, slots.numel()))
        if self.rope.rot_dim:
            expect(positions, "positions", torch.int32, dev, max(n_tok, positions.numel()))
            expect(self.freqs, "freqs", torch.int64, dev, self.rope.rot_dim // 2)
        for x, what in ((self.wq, "wq"), (self.wk, "wk")):
            if x is not None:
                expect(x, what, self.dtype, dev, c.head_dim)
        step = qkv.stride(0) if n_tok > 1 else qkv.shape[1]      # (of a single row torch may report any)
        q = qkv.data_ptr()
        k = q + c.n_q_heads * c.head_dim * qkv.element_size()
        v = k + c.n_kv_heads * c.head_dim * qkv.element_size()
        kc, vc = pool.k_cache[layer], pool.v_cache[layer]
        with OnStream(stream, qkv, slots, positions, self.wq, self.wk, self.freqs, kc, vc) as on:
            out = torch.empty((n_tok, c.n_q_heads, c.head_dim), dtype=qkv.dtype, device=dev)
            H.hybrid_qk_norm_rope_cache(c, self.rope, pool.pg, q, step, k, step, v, step, n_tok, self.wq, self.wk, positions,
                                        self.freqs, slots, out, kc, vc)
            return on.returns(out)

    def attend(self, q, pool: PagePool, layer: int, stream=None, rows: BlockRows | None = None):
        """Queries of the active blocks against the cache -> the same shape.

        q [n_req * B, Hq, d]: token i of request r in row r * B + i, so that every request has B tokens. With rows
        (pool.block_rows), q [n_tok, Hq, d] is packed by request as pool.append packs it; outputs beyond the last token
        are zeros, and of a request's tokens beyond its first B NaN: attention has no row for them."""
        self._check_pool(pool)
        c, n_rows = self.cfg, pool.n_req * self.cfg.block_size
        if rows is None:
            lead = q.shape[:-2] if math.prod(q.shape[:-2]) == n_rows else (n_rows,)
        elif rows.n_rows != n_rows:
            raise ValueError(f"rows: made for {rows.n_rows} query rows, not for {n_rows}")
        else:
            lead = (rows.n_tok,)
        expect(q, "q", self.dtype, pool.device, *lead, c.n_q_heads, c.head_dim)
        kc, vc = pool.k_cache[layer], pool.v_cache[layer]
        with OnStream(stream, q, kc, vc, pool.block_table, pool.lens) as on:
            if rows is None:
                out = torch.empty_like(q)
            elif rows.n_tok == 0:
                return on.returns(torch.empty_like(q))
            else:
                on.uses(rows.token, rows.row, pool.no_row)
                q = q.index_select(0, rows.token)
                out = torch.empty((n_rows + 2, *q.shape[1:]), dtype=q.dtype, device=q.device)
                out[n_rows:].copy_(pool.no_row)
            workspace = pool.workspace_of(c, on)
            H.hybrid_paged_attn(c, pool.pg, q, kc, vc, pool.block_table, pool.lens, pool.n_req, self.window, self.n_sink,
                                out, workspace, workspace.numel())
            return on.returns(out if rows is None else out.index_select(0, rows.row))

    def step(self, qkv, pool: PagePool, layer: int, slots, positions, stream=None, rows: BlockRows | None = None):
        """One denoising step of the active blocks (or, with B = 1, one token); rows: see attend."""
        return self.attend(self.write(qkv, pool, layer, slots, positions, stream), pool, layer, stream, rows)
