"""The checks of the pool and the layer of the softmax layers on the host: what does not fit is refused before
the library is called."""
import pytest
import torch

from paper_2608_06628_gb300 import build as B
from paper_2608_06628_gb300 import hybrid as H
from paper_2608_06628_gb300.page_pool import PagePool
from paper_2608_06628_gb300.softmax_layer import SoftmaxLayer

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HQ, HKV, D, BS, N = 4, 2, 64, 2, 3
WIDTH = (HQ + 2 * HKV) * D


@pytest.fixture(scope="module", autouse=True)
def _library():
    B.build()


@pytest.fixture
def calls(monkeypatch):
    """The entry points that were reached, with their arguments."""
    seen = []
    for name in ("hybrid_page_append", "hybrid_page_release", "hybrid_qk_norm_rope_cache", "hybrid_paged_attn"):
        monkeypatch.setattr(H, name, lambda *a, _name=name, **kw: seen.append((_name, a)))
    monkeypatch.setattr(H, "_stream", lambda stream: 0 if stream is None else stream)
    return seen


def cfg(d=D, Hq=HQ, Hkv=HKV, Bs=BS, dt=F32):
    return H.make_cfg(d, 64, Hq, Hkv, Bs, dt)


def pool(**kw):
    return PagePool(cfg(**kw), N, 20, 64, 16, device="cpu")


def layer(c=None, rot=D, **kw):
    return SoftmaxLayer(c or cfg(), H.make_rope(rot, device="cpu"), **kw)


def ints(n, dtype=I32):
    return torch.zeros(n, dtype=dtype)


def wide(n):
    """Every second entry of twice as many."""
    return torch.zeros(2 * n, dtype=I32)[::2]


@pytest.mark.parametrize("n_new", [ints(N, torch.int64), ints(N - 1), ints(N + 1), wide(N), ints(N).view(1, N), torch.zeros(N), [1, 2, 3]])
def test_append_refuses(calls, n_new):
    with pytest.raises(ValueError, match="n_new"):
        pool().append(n_new, 6)
    assert not calls


@pytest.mark.parametrize("rows", [ints(2, torch.int64), wide(2), ints(2).view(2, 1), torch.zeros(2), torch.zeros(2, dtype=torch.bool)])
def test_release_refuses(calls, rows):
    with pytest.raises(ValueError, match="rows"):
        pool().release(rows)
    assert not calls


@pytest.mark.parametrize("what,kw", [
    ("qkv", dict(qkv=torch.zeros(6, WIDTH, dtype=BF))), ("qkv", dict(qkv=torch.zeros(6, WIDTH + 1))),
    ("qkv", dict(qkv=torch.zeros(WIDTH, 6).t())), ("qkv", dict(qkv=torch.zeros(1, 6, WIDTH))), ("qkv", dict(qkv=torch.zeros(WIDTH))),
    ("slots", dict(slots=ints(6, torch.int64))), ("slots", dict(slots=ints(5))), ("slots", dict(slots=wide(6))),
    ("positions", dict(positions=ints(6, torch.int64))), ("positions", dict(positions=ints(5))),
    ("positions", dict(positions=wide(6))),
])
def test_write_refuses(calls, what, kw):
    args = dict(qkv=torch.zeros(6, WIDTH), slots=ints(6), positions=ints(6))
    with pytest.raises(ValueError, match=what):
        layer().write(pool=pool(), layer=0, **{**args, **kw})
    assert not calls


@pytest.mark.parametrize("what,kw", [("wq", dict(wq=torch.ones(D, dtype=BF))), ("wk", dict(wk=torch.ones(D + 1))),
                                     ("wq", dict(wq=torch.ones(2 * D)[::2]))])
def test_write_refuses_weights(calls, what, kw):
    with pytest.raises(ValueError, match=what):
        layer(**kw).write(torch.zeros(6, WIDTH), pool(), 0, ints(6), ints(6))
    assert not calls


@pytest.mark.parametrize("q", [torch.zeros(N * BS - 1, HQ, D), torch.zeros(N * BS + 1, HQ, D), torch.zeros(N * BS, HQ, D, dtype=BF),
                               torch.zeros(N * BS, D, HQ).transpose(1, 2), torch.zeros(N * BS, HQ, 2 * D)[..., :D],
                               torch.zeros(N * BS, HQ * D), torch.zeros(0, HQ, D)])
def test_attend_refuses(calls, q):
    with pytest.raises(ValueError, match="q:"):
        layer().attend(q, pool(), 0)
    assert not calls


def test_step_refuses_part_of_a_batch(calls):
    with pytest.raises(ValueError, match="q:"):
        layer().step(torch.zeros(4, WIDTH), pool(), 0, ints(4), ints(4))


def test_what_fits_goes_through(calls):
    p = pool()
    p.append(ints(N), 6)
    p.release(ints(0))
    out = layer(wq=torch.ones(D), wk=torch.ones(D)).write(torch.zeros(6, WIDTH + 8)[:, :WIDTH], p, 0, ints(9), ints(6))
    assert out.shape == (6, HQ, D) and calls[-1][0] == "hybrid_qk_norm_rope_cache" and calls[-1][1][4] == WIDTH + 8
    # one row, of which torch may report any stride; nothing rotated, so no positions
    layer(rot=0).write(torch.zeros(WIDTH).expand(1, WIDTH), p, 0, ints(1), None)
    assert calls[-1][1][4] == calls[-1][1][6] == calls[-1][1][8] == WIDTH
    layer().write(torch.zeros(0, WIDTH), p, 0, ints(0), ints(0))
    for lead in ((N * BS,), (N, BS)):
        assert layer().attend(torch.zeros(*lead, HQ, D), p, 0).shape == (*lead, HQ, D)
    assert [name for name, _ in calls].count("hybrid_paged_attn") == 2


@pytest.mark.parametrize("new,n_tok", [([2, 0, 2], 4), ([2, 0, 2], 6), ([0, 1, 0], 1), ([1, 2, 1], 9), ([0, 0, 0], 3), ([0, 0, 0], 0),
                                       ([3, 0, 5], 8), ([2, 2, 2], 6)])
def test_packed_tokens_and_query_rows(calls, monkeypatch, new, n_tok):
    """Attention that returns its queries: every token gets its own back, from the row of its request."""
    taken = []

    def same(cfg, pg, q, *args, **kw):
        taken.append(q.clone())
        args[7][:q.shape[0]] = q

    monkeypatch.setattr(H, "hybrid_paged_attn", same)
    p, offs = pool(), torch.tensor([0, *torch.tensor(new).cumsum(0).tolist()], dtype=I32)
    rows = p.block_rows(offs, n_tok)
    q = (torch.arange(n_tok * HQ * D, dtype=F32) + 1).view(n_tok, HQ, D)
    out = layer().attend(q, p, 0, rows=rows)
    assert out.shape == q.shape and len(taken) == (n_tok > 0)
    t = 0
    for r, n in enumerate(new):
        for i in range(n):
            if i < BS:
                assert torch.equal(out[t], q[t]) and torch.equal(taken[0][r * BS + i], q[t])
            else:
                assert bool(out[t].isnan().all())
            t += 1
    assert not bool(out[t:].any())


def test_packed_rows_refused(calls):
    p, offs = pool(), torch.tensor([0, 2, 4, 6], dtype=I32)
    for bad in (offs.long(), offs[:3], torch.zeros(8, dtype=I32)[::2]):
        with pytest.raises(ValueError, match="offsets"):
            p.block_rows(bad, 6)
    with pytest.raises(ValueError, match="rows"):
        layer().attend(torch.zeros(6, HQ, D), p, 0, rows=p.block_rows(offs, 6, 5))
    with pytest.raises(ValueError, match="q:"):
        layer().attend(torch.zeros(5, HQ, D), p, 0, rows=p.block_rows(offs, 6))
    assert not calls


def test_offsets_out_of_range_index_nothing(calls):
    """Offsets that no append gives (they are the caller's memory) stay within the tensors."""
    p = pool()
    for offs in ([0, 900, -5, 2 ** 31 - 1], [-9, -7, -3, -1], [2 ** 31 - 1, 0, 0, 4]):
        rows = p.block_rows(torch.tensor(offs, dtype=I32), 6)
        assert 0 <= int(rows.token.min()) and int(rows.token.max()) < 6 and 0 <= int(rows.row.min()) and int(rows.row.max()) <= N * BS + 1


@pytest.mark.parametrize("kw", [dict(d=128), dict(Hkv=4), dict(Hkv=1), dict(dt=BF)])
def test_a_layer_of_other_caches_than_the_pools_is_refused(calls, kw):
    """More key heads, or a wider type, would write beyond the pool's caches."""
    c = cfg(**kw)
    width, dt = (c.n_q_heads + 2 * c.n_kv_heads) * c.head_dim, kw.get("dt", F32)
    lay = SoftmaxLayer(c, H.make_rope(c.head_dim, device="cpu"))
    with pytest.raises(ValueError, match="pool"):
        lay.write(torch.zeros(6, width, dtype=dt), pool(), 0, ints(6), ints(6))
    with pytest.raises(ValueError, match="pool"):
        lay.attend(torch.zeros(6, c.n_q_heads, c.head_dim, dtype=dt), pool(), 0)
    assert not calls


@pytest.mark.parametrize("kw", [dict(Bs=1), dict(Bs=64), dict(Hq=8), dict(Hq=2)])
def test_a_layer_with_other_rows_than_the_pools_is_taken(calls, kw):
    c = cfg(**kw)
    SoftmaxLayer(c, H.make_rope(64, device="cpu")).attend(torch.zeros(N * c.block_size, c.n_q_heads, D), pool(), 0)
    (name, args), = calls
    assert name == "hybrid_paged_attn" and args[11].numel() == args[12] == H.hybrid_paged_attn_workspace_bytes(c, pool().pg, N)
