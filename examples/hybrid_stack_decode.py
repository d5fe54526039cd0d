"""Blockwise decoding of a hybrid stack: softmax layers over a paged cache beside block-hybrid
layers with a fixed-size state, for a batch of requests with prompts of different lengths.

    python examples/hybrid_stack_decode.py [--requests 64] [--blocks 4] [--steps 8]

The projections, the MLPs and the sampling of a model are stood in for by random qkv of their
shape; every layer of attention runs in full:

  prompt   pool.append; each softmax layer writes its keys and values to the cache, each hybrid
           layer folds its keys and values into its state (hybrid_commit_ragged)
  block    pool.append for B tokens of each request, then per denoising step
             softmax layer  norm + rotation + cache write, attention over prefix and block
             hybrid layer   norm + rotation, block-hybrid step
           and the last step commits the block to the states
  end      the pages of half of the requests go back to the pool

Prints the time of a denoising step of the whole stack, and checks one softmax layer's last
output against float64 attention over its cache.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_06628_gb300 import hybrid as H  # noqa: E402
from paper_2608_06628_gb300.page_pool import PagePool  # noqa: E402
from paper_2608_06628_gb300.softmax_layer import SoftmaxLayer  # noqa: E402
from paper_2608_06628_gb300.state_pool import StatePool  # noqa: E402


def check_softmax_layer(q, out, pool, layer, scale):
    """Worst rel-L2 over requests of out against float64 softmax over the whole cache of each."""
    P, worst = pool.pg.page_size, 0.0
    G = q.shape[2] // pool.cfg.n_kv_heads
    for r, n in enumerate(pool.lens.tolist()):
        j = torch.arange(n, device=q.device)
        page = pool.block_table[r][j // P].long()
        k = pool.k_cache[layer][page, :, j % P].double().repeat_interleave(G, 1)
        v = pool.v_cache[layer][page, :, j % P].double().repeat_interleave(G, 1)
        p = torch.softmax(torch.einsum("bhd,khd->bhk", q[r].double(), k) * scale, -1)
        want = torch.einsum("bhk,khd->bhd", p, v)
        worst = max(worst, float((out[r].double() - want).norm() / want.norm()))
    return worst


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=64)
    ap.add_argument("--prompt-max", type=int, default=2048)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--softmax-layers", type=int, default=2)
    ap.add_argument("--hybrid-layers", type=int, default=1)
    a = ap.parse_args(argv)
    n, B, Hq, Hkv, d, F, page = a.requests, 32, 16, 4, 128, 128, 32
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(0)
    randn = lambda *s: torch.randn(s, generator=gen, device=dev).to(torch.bfloat16)  # noqa: E731
    cfg = H.make_cfg(d, F, Hq, Hkv, B, torch.bfloat16)

    max_len = a.prompt_max + a.blocks * B
    pool = PagePool(cfg, n, n * (-(-max_len // page)), max_len, page, a.softmax_layers, dev)
    rope = H.make_rope(d, base=10000.0, kind=H.HYBRID_ROPE_YARN, factor=4.0, device=dev)
    layers = [SoftmaxLayer(cfg, rope, 1 + 0.1 * randn(d), 1 + 0.1 * randn(d)) for _ in range(a.softmax_layers)]
    norm = SoftmaxLayer(cfg, rope, 1 + 0.1 * randn(d), 1 + 0.1 * randn(d))     # of the hybrid layers
    states = [StatePool(cfg, n, dev) for _ in range(a.hybrid_layers)]
    ptrs = [s.all_ptrs() for s in states]
    W, alpha = (randn(Hkv, d, F).float() / math.sqrt(d)).to(torch.bfloat16), torch.rand(Hq, generator=gen, device=dev)
    for p in ptrs:
        H.hybrid_state_init(cfg, p, n)

    def rotated(qkv, positions):
        q, k, v = norm.split(qkv)
        qo, ko = torch.empty(q.shape, dtype=q.dtype, device=dev), torch.empty(k.shape, dtype=k.dtype, device=dev)
        H.hybrid_qk_norm_rope(cfg, norm.rope, q, q.stride(0), k, k.stride(0), q.shape[0], norm.wq, norm.wk, positions,
                              norm.freqs, qo, ko)
        return qo, ko, v.contiguous()

    # prompts
    lens = torch.randint(1, a.prompt_max + 1, (n,), generator=gen, device=dev, dtype=torch.int32)
    total = int(lens.sum())
    slots, positions, offsets = pool.append(lens, total)
    for i, layer in enumerate(layers):
        layer.write(randn(total, (Hq + 2 * Hkv) * d), pool, i, slots, positions)
    for p in ptrs:
        _, k, v = rotated(randn(total, (Hq + 2 * Hkv) * d), positions)
        H.hybrid_commit_ragged(cfg, k, v, offsets.tolist(), W, p, n)
    H.hybrid_check()

    # blocks
    qkv = [randn(n * B, (Hq + 2 * Hkv) * d) for _ in range(len(layers) + len(ptrs))]
    block = torch.full((n,), B, dtype=torch.int32, device=dev)
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for b in range(a.blocks):
        slots, positions, _ = pool.append(block, n * B)
        for s in range(a.steps):
            if (b, s) == (a.blocks - 1, 0):
                start.record()
            for i, layer in enumerate(layers):
                q = layer.write(qkv[i], pool, i, slots, positions)
                out = layer.attend(q, pool, i)
            for i, p in enumerate(ptrs):
                qo, ko, v = rotated(qkv[len(layers) + i], positions)
                o = torch.empty_like(qo)
                step = H.hybrid_block_attn_commit if s == a.steps - 1 else H.hybrid_block_attn
                step(cfg, qo, ko, v, W, alpha, p, n, o)
    end.record()
    H.hybrid_check()
    err = check_softmax_layer(q.view(n, B, Hq, d), out.view(n, B, Hq, d), pool, len(layers) - 1, 1 / math.sqrt(d))
    pool.release(torch.arange(0, n, 2, dtype=torch.int32, device=dev))
    H.hybrid_check()
    us = start.elapsed_time(end) * 1e3 / a.steps
    print(f"{n} requests, {int(pool.lens.sum())} tokens left in the cache, {int(pool.ring[1])} of {pool.pg.n_pages} pages free")
    print(f"denoising step of {len(layers)} softmax and {len(ptrs)} hybrid layers: {us:.1f} us; "
          f"softmax layer against float64: rel-L2 {err:.2e}")
    assert err <= 1e-2 and bool(torch.isfinite(o.float()).all())
    return us, err


if __name__ == "__main__":
    main()
