"""Paged key-value caches of a model's softmax layers, and the tables that all layers share.

The device holds everything: lengths, block table and the ring of free pages are
int32 tensors that hybrid_page_append and hybrid_page_release read and write, so a
serving loop never waits for the host to count pages.  Those calls read one copy of
lengths and ring and write another, which the pool copies back: its tensors stay
the same ones, and a captured graph may hold any number of calls.  Rows of the table
are the requests of the batch; a released row may take a new request at once.
"""
from __future__ import annotations

import contextlib
import math

import torch

from . import hybrid as H


def expect(x, what: str, dtype, device, *shape, rows=False):
    """ValueError unless x is a tensor of that type and shape on that device: dense, or (rows) with dense rows."""
    if isinstance(x, torch.Tensor) and x.dtype == dtype and tuple(x.shape) == shape and x.device == device and \
            (x.is_contiguous() or (rows and x.stride(-1) == 1)):
        return
    has = f"{x.dtype} {list(x.shape)}, strides {x.stride()}, on {x.device}" if isinstance(x, torch.Tensor) else type(x).__name__
    raise ValueError(f"{what}: {has} where a dense {dtype} {list(shape)} on {device} is wanted")


class OnStream:
    """A call's work on its stream (None: the current one; else torch's stream or a raw handle): torch's own kernels
    and allocations go there too. `used` is what the work reads and writes besides: its memory is not handed out again
    before the work is done, whenever the caller drops it, and what returns() is given not before the caller's stream is
    done with it. The order between the two streams (events, wait_stream) is the caller's."""

    def __init__(self, stream, *used):
        if stream is None:
            self.caller, self.scope = None, contextlib.nullcontext()
            return
        if not isinstance(stream, torch.cuda.Stream):
            handle = stream if isinstance(stream, int) else stream.cuda_stream
            # 0 and 1 (cudaStreamLegacy) both name the default stream
            stream = torch.cuda.ExternalStream(handle) if handle > 1 else torch.cuda.default_stream()
        self.caller, self.scope = torch.cuda.current_stream(), torch.cuda.stream(stream)
        self.stream = stream
        self.uses(*used)

    def __enter__(self):
        self.scope.__enter__()
        return self

    def __exit__(self, *exc):
        return self.scope.__exit__(*exc)

    def uses(self, *used):
        if self.caller is not None:
            for x in used:
                if x is not None:
                    x.record_stream(self.stream)

    def returns(self, *made):
        if self.caller is not None:
            for x in made:
                x.record_stream(self.caller)
        return made[0] if len(made) == 1 else made


class BlockRows:
    """Where the packed tokens of an append stand among the n_req * B query rows of attention, whose row r * B + i is
    token i of request r: for batches where a request has fewer than B new tokens, or none."""

    def __init__(self, offsets, n_req: int, n_tok: int, block: int):
        self.n_tok, self.n_rows, dev = n_tok, n_req * block, offsets.device
        t = torch.arange(max(n_tok, block), dtype=torch.int32, device=dev)
        # rows without a token repeat one: nothing reads what they give
        self.token = (offsets[:-1, None] + t[:block]).view(-1).clamp_(0, max(n_tok - 1, 0))
        t = t[:n_tok]
        r = torch.searchsorted(offsets[1:], t, right=True, out_int32=True)
        i = t - offsets.index_select(0, r)
        # the row of a token; beyond its request's first B tokens n_rows + 1, beyond the last token n_rows
        row = torch.where(i < block, torch.add(i, r, alpha=block), self.n_rows + 1)
        self.row = torch.where(r < n_req, row, self.n_rows).clamp_(0, self.n_rows + 1)


class PagePool:
    def __init__(self, cfg: H.hybrid_cfg, n_req: int, n_pages: int, max_len: int, page_size: int = 32, n_layers: int = 1,
                 device="cuda"):
        self.cfg, self.n_req, self.n_layers = cfg, n_req, n_layers
        self.pg = H.make_page_cfg(page_size, n_pages, -(-max_len // page_size))
        dtype = torch.bfloat16 if cfg.io_dtype == H.HYBRID_BF16 else torch.float32
        shape = (n_layers, n_pages, cfg.n_kv_heads, page_size, cfg.head_dim)
        self.k_cache = torch.empty(shape, dtype=dtype, device=device)
        self.v_cache = torch.empty(shape, dtype=dtype, device=device)
        self.device = self.k_cache.device
        self.block_table = torch.full((n_req, self.pg.max_pages), -1, dtype=torch.int32, device=device)
        self.free_pages = torch.arange(n_pages, dtype=torch.int32, device=device)
        # {head, count} of the ring, the lengths, and an entry that release() writes for rows that are not there; then
        # the same as calls write it
        self._state = torch.zeros(2, n_req + 3, dtype=torch.int32, device=device)
        self._state[:, 1] = n_pages
        now, then = self._state
        self._now, self._then, self._ring, self._lens = now[:-1], then[:-1], now[:2], now[2:-1]
        self._then_ring, self._then_lens, self._lens_and_spare = then[:2], then[2:-1], now[2:]
        self.workspace_bytes = H.hybrid_paged_attn_workspace_bytes(cfg, self.pg, n_req)
        if self.workspace_bytes == 0:
            raise ValueError(f"unsupported {cfg} with {self.pg}")
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device=device)
        self._workspaces = {}
        # outputs of tokens without a query row: beyond the last token, beyond a request's first block of them
        self.no_row = torch.tensor([[[0.0]], [[math.nan]]], dtype=dtype, device=device)

    @property
    def lens(self) -> torch.Tensor:
        """Tokens of each request, int32 [n_req]."""
        return self._lens

    @property
    def ring(self) -> torch.Tensor:
        """{head, count} of the free pages."""
        return self._ring

    def _tables(self):
        return self._state, self.block_table, self.free_pages

    def workspace_of(self, cfg: H.hybrid_cfg, on: OnStream) -> torch.Tensor:
        """Attention's workspace for a layer's cfg on the call's stream: calls on several streams may overlap, and need
        one each. A captured call has one of its graph's memory, since the graph may be replayed beside any of them."""
        key = (H._stream(None), cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads, cfg.block_size, cfg.io_dtype)
        capturing = self.device.type == "cuda" and torch.cuda.is_current_stream_capturing()
        made = None if capturing else self._workspaces.get(key)
        if made is None:
            n = H.hybrid_paged_attn_workspace_bytes(cfg, self.pg, self.n_req)
            if n == 0:
                raise ValueError(f"unsupported {cfg} with {self.pg}")
            if not capturing and not self._workspaces and n == self.workspace_bytes:
                made = self.workspace
            else:
                made = torch.empty(n, dtype=torch.uint8, device=self.device)
            if not capturing:
                self._workspaces[key] = made
        on.uses(made)
        return made

    def append(self, n_new: torch.Tensor, n_tok: int, stream=None):
        """Room for n_new [n_req] (int32, device) more tokens of each request, at most n_tok in all.
        Returns slots, positions [n_tok] and tok_offsets [n_req + 1] (int32); slots beyond the last
        token, and of requests that did not fit (see hybrid_check), are -1. Tokens are packed by request:
        see block_rows where not every request has a whole block of them."""
        expect(n_new, "n_new", torch.int32, self.device, self.n_req)
        new = lambda n: torch.empty(n, dtype=torch.int32, device=self.device)  # noqa: E731
        with OnStream(stream, n_new, *self._tables()) as on:
            slots, positions, offsets = new(n_tok), new(n_tok), new(self.n_req + 1)
            H.hybrid_page_append(self.pg, self.n_req, self._lens, n_new, self.free_pages, self._ring, self.block_table, slots,
                                 positions, n_tok, offsets, self._then_lens, self._then_ring)
            self._now.copy_(self._then)
            return on.returns(slots, positions, offsets)

    def block_rows(self, offsets: torch.Tensor, n_tok: int, block: int | None = None, stream=None) -> BlockRows:
        """For SoftmaxLayer.attend and step, once per append: which query row each of its n_tok packed tokens has.
        offsets: the append's tok_offsets; block: the layers' block size (None: the pool's)."""
        expect(offsets, "offsets", torch.int32, self.device, self.n_req + 1)
        with OnStream(stream, offsets) as on:
            rows = BlockRows(offsets, self.n_req, n_tok, block or self.cfg.block_size)
            on.returns(rows.token, rows.row)
            return rows

    def release(self, rows: torch.Tensor, stream=None):
        """Give back the pages of the requests in rows (int32, device, each once); their lengths become 0, on the
        same stream. A row out of range is left out, and reported by hybrid_check."""
        expect(rows, "rows", torch.int32, self.device, rows.numel())
        with OnStream(stream, rows, *self._tables()):
            H.hybrid_page_release(self.pg, self.n_req, rows, rows.numel(), self._lens, self.block_table, self.free_pages,
                                  self._ring, self._then_ring)
            self._ring.copy_(self._then_ring)
            # rows below 0 and above the last all become the entry behind the lengths (-1 counts from the end)
            self._lens_and_spare.index_fill_(0, rows.long().clamp_(-1, self.n_req), 0)
