"""Paged attention in bfloat16 at the numbers of rows where the tensor-core kernel changes its layout, and what cache
writes leave alone.  The bounds are those of test_gpu_softmax.py."""
import pytest
import torch

from paper_2608_06628_gb300 import hybrid as H
from test_gpu_softmax import EDGES, _device, attn_setup, check_attn, gen, rope_setup, run_rope  # noqa: F401

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,G", [(31, 1), (8, 4), (33, 1), (3, 11), (41, 1), (63, 1), (16, 4), (13, 5), (33, 2), (19, 5), (24, 4), (97, 1),
                                 (14, 7), (127, 1), (43, 3)])
def test_attention_rows_of_a_tile(B, G, d):
    """1 to 4 quarters of Tensor Memory at work, in 4, 2 and 1 copies; masks of both kinds, requests that are split."""
    for window, sink, scale in ((0, 0, 1.0), (300, 5, 4.0), (1000, 130, 1.0)):
        s = attn_setup(BF, B, 3 * G, 3, d, 16, EDGES + [9003], window, sink, seed=B + 20 * G, k_scale=scale)
        check_attn(s, f"{B} tokens, {G} heads to a key head, window {window}")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,d,P", [(5, 16, 4, 128, 32), (700, 6, 3, 64, 128)])
def test_cache_writes_leave_the_rest_alone(dt, T, Hq, Hkv, d, P):
    """Slots beyond the pool and padding write nothing, the tokens beside them go where they belong."""
    s = rope_setup(T, Hq, Hkv, d, d, dt, seed=T)
    n_pages = -(-T // P) + 2
    slots = torch.randperm(n_pages * P, generator=gen(2), device="cuda")[:T].to(torch.int32)
    slots[1] = -1
    for t, x in ((0, n_pages * P), (2, 2 ** 31 - 1), (T // 2, n_pages * P + 5), (T - 1, -2 ** 31)):
        slots[t] = x
    kc, vc = (torch.full((n_pages, Hkv, P, d), x, dtype=dt, device="cuda") for x in (7.0, 8.0))
    want_k, want_v = kc.clone(), vc.clone()
    qo, ko = run_rope(s)
    live = (slots >= 0) & (slots < n_pages * P)
    at = slots[live].long()
    want_k[at // P, :, at % P] = ko[live]
    want_v[at // P, :, at % P] = s["v"][live]
    q = torch.empty_like(qo)
    H.hybrid_qk_norm_rope_cache(s["cfg"], s["rope"], H.make_page_cfg(P, n_pages, 1), s["q"], s["stride"], s["k"], s["stride"],
                                s["v"], s["stride"], T, s["wq"], s["wk"], s["pos"], s["freqs"], slots, q, kc, vc)
    assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
    assert torch.equal(q, qo) and torch.equal(kc, want_k) and torch.equal(vc, want_v)
