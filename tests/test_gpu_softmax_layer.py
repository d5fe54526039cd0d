"""The pool and the layer of the softmax layers as a serving loop uses them: streams, batches with idle
rows, graphs, and infinities in the cache."""
import pytest
import torch

import softmax_reference as R
from gpu_harness import assert_parity
from paper_2608_06628_gb300 import hybrid as H
from paper_2608_06628_gb300.page_pool import PagePool
from paper_2608_06628_gb300.softmax_layer import SoftmaxLayer

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_06628_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def late(stream):
    """What is queued on the stream from here on starts about a tenth of a second later."""
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)


def pool_of(new, n_pages=20, cfg=None, max_len=64):
    cfg = cfg or H.make_cfg(64, 64, 2, 1, 4, F32)
    pool = PagePool(cfg, len(new), n_pages, max_len, 16)
    pool.append(i32(new), sum(new))
    H.hybrid_check()
    return pool


# ------------------------------------------------------------------ streams

@pytest.mark.parametrize("raw", [False, True])
def test_release_on_another_stream(raw):
    """The lengths are reset after the release has read them, wherever it runs."""
    s = torch.cuda.Stream()
    rows = i32([1])
    pool_of([20, 33, 5]).release(rows, stream=s)             # its kernels are loaded, which may wait for the GPU
    pool = pool_of([20, 33, 5])
    late(s)
    pool.release(rows, stream=s.cuda_stream if raw else s)
    torch.cuda.synchronize()
    H.hybrid_check()
    assert pool.ring.tolist() == [6, 17] and pool.lens.tolist() == [20, 0, 5]


def test_release_on_the_default_stream_by_its_handle():
    pool = pool_of([20, 33, 5])
    pool.release(i32([0, 2]), stream=0)
    H.hybrid_check()
    assert pool.ring.tolist() == [6, 17] and pool.lens.tolist() == [0, 33, 0]


@pytest.mark.parametrize("handle", [1, 2])
def test_release_on_the_runtimes_special_handles(handle):
    """cudaStreamLegacy and cudaStreamPerThread, as the C entry points take them."""
    pool = pool_of([20, 33, 5])
    rows = i32([0, 2])
    torch.cuda.synchronize()
    pool.release(rows, stream=handle)
    torch.cuda.synchronize()
    H.hybrid_check()
    assert pool.ring.tolist() == [6, 17] and pool.lens.tolist() == [0, 33, 0]


@pytest.mark.parametrize("rows,lens,free", [([-1], [20, 33, 5], 14), ([3], [20, 33, 5], 14), ([2 ** 31 - 1, 1, -2 ** 31], [20, 0, 5], 17),
                                            ([], [20, 33, 5], 14)])
def test_release_leaves_out_rows_that_are_not_there(rows, lens, free):
    pool = pool_of([20, 33, 5])
    pool.release(i32(rows))
    bad = any(not 0 <= r < 3 for r in rows)
    assert H.hybrid_check(check=False) == (H.HYBRID_ERR_DEVICE if bad else H.HYBRID_OK)
    assert pool.lens.tolist() == lens and pool.ring.tolist() == [6, free]
    pool.append(i32([3, 4, 2]), 9)
    H.hybrid_check()
    assert pool.lens.tolist() == [x + y for x, y in zip(lens, [3, 4, 2])]


def layer_of(pool, **kw):
    return SoftmaxLayer(pool.cfg, H.make_rope(pool.cfg.head_dim), **kw)


def same_call(make):
    """make(stream) on a late stream, its arguments and results dropped before it has run, while the current
    stream takes memory of every size that they had: returns what the call gives on the current stream, on
    the late one, and whether the other memory kept what was written to it."""
    s = torch.cuda.Stream()
    make(s)
    want = [x.clone() for x in make(None)]
    torch.cuda.synchronize()
    late(s)
    got = make(s)
    kept = []
    with torch.cuda.stream(s):
        kept = [x.clone() for x in got]                      # of the late stream, behind the call
    sizes = [x.nbytes for x in got]
    del got
    other = [torch.full((n // 4,), 55, dtype=torch.int32, device="cuda") for n in sizes for _ in range(4)]
    torch.cuda.synchronize()
    H.hybrid_check()
    return want, kept, all(bool((x == 55).all()) for x in other)


def test_append_on_another_stream_keeps_its_memory():
    new = [1000, 1000, 48]

    def append(stream):
        pool = PagePool(H.make_cfg(64, 64, 2, 1, 4, F32), 3, 400, 4096, 16)
        torch.cuda.current_stream().synchronize()
        n_new = i32(new)
        got = pool.append(n_new, 2048, stream=stream)
        del n_new
        torch.zeros(3, dtype=torch.int32, device="cuda")     # in the place of n_new, where that is free
        return (*got, pool.lens)

    want, got, intact = same_call(append)
    assert intact and all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dt", [BF, F32])
def test_layer_on_another_stream_keeps_its_memory(dt):
    cfg = H.make_cfg(64, 64, 4, 2, 2, dt)
    pool = pool_of([300, 200, 100], 60, cfg, 400)
    pool.k_cache.normal_()
    pool.v_cache.normal_()
    layer = layer_of(pool)
    slots, positions, _ = pool.append(i32([2, 2, 2]), 6)
    x = torch.randn(6, 8 * 64, device="cuda").to(dt)
    torch.cuda.synchronize()

    def step(stream):
        q = layer.write(x.clone(), pool, 0, slots.clone(), positions.clone(), stream)
        torch.zeros_like(x), torch.zeros_like(slots), torch.zeros_like(slots)    # in the place of the copies
        return q, layer.attend(q, pool, 0, stream), layer.step(x, pool, 0, slots, positions, stream)

    # (the copies are made on the current stream, which has to be done before the late one begins: it is late)
    want, got, intact = same_call(step)
    assert intact and all(torch.equal(a, b) for a, b in zip(got, want))


def filled(cfg, new, n_pages, max_len):
    pool = pool_of(new, n_pages, cfg, max_len)
    pool.k_cache.normal_()
    pool.v_cache.normal_()
    return pool


def test_streams_have_workspaces_of_their_own(monkeypatch):
    cfg = H.make_cfg(64, 64, 4, 2, 2, BF)
    pool = filled(cfg, [300, 200, 100], 60, 400)
    layer, q = layer_of(pool), torch.randn(6, 4, 64, device="cuda").to(BF)
    seen, call = [], H.hybrid_paged_attn

    def note(*args, **kw):
        seen.append(args[11].data_ptr())
        return call(*args, **kw)

    monkeypatch.setattr(H, "hybrid_paged_attn", note)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (None, a, b, a, None, b):
        layer.attend(q, pool, 0, s)
    H.hybrid_check()
    assert len(set(seen[:3])) == 3 and seen[3:] == [seen[1], seen[0], seen[2]]


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_on_two_streams_at_once(dt):
    """Contexts that are split over many blocks, so that every call has partial results in its workspace."""
    cfg = H.make_cfg(128, 64, 8, 2, 16, dt)
    pool = filled(cfg, [9000, 20000, 700], 1900, 20000)
    layer = layer_of(pool)
    q = [torch.randn(48, 8, 128, device="cuda").to(dt) for _ in range(2)]
    want = [layer.attend(x, pool, 0) for x in q]
    streams = [torch.cuda.Stream() for _ in q]
    torch.cuda.synchronize()
    got = [layer.attend(q[i], pool, 0, streams[i]) for _ in range(20) for i in range(2)]
    torch.cuda.synchronize()
    H.hybrid_check()
    assert all(torch.equal(x, want[i % 2]) for i, x in enumerate(got))


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_of_layers_with_other_rows_than_the_pool(dt):
    """The pool is made for single tokens of 4 heads; the layer asks for blocks of 33 of 6 heads."""
    pool = filled(H.make_cfg(64, 64, 4, 2, 1, dt), [300, 0, 5000], 400, 5000)
    layer = SoftmaxLayer(H.make_cfg(64, 64, 6, 2, 33, dt), H.make_rope(64))
    q = torch.randn(99, 6, 64, device="cuda").to(dt)
    got = layer.attend(q, pool, 0)
    H.hybrid_check()
    want = R.paged_attention(q.view(3, 33, 6, 64), pool.k_cache[0], pool.v_cache[0], pool.block_table, pool.lens.tolist(), 0, 0)
    assert_parity(got.view(want.shape).double().cpu().numpy(), want.cpu().numpy(), dt, "blocks of 33", units="out")


# ------------------------------------------------------------------ entries that are no pages

@pytest.mark.parametrize("n,pages,bad", [(1, 3, [0]), (3, 3, [2, 5]), (2, 400, [0, 255, 256, 700]), (300, 40, range(0, 12000, 7)),
                                         (7, 100, range(700)), (5, 60, [])])
def test_release_leaves_out_entries_that_are_no_pages(n, pages, bad):
    """They stay out of the ring, the pages beside them go into it in order, and the calls behind are whole again."""
    P, N = 16, n * pages + 9
    order = torch.randperm(N, generator=torch.Generator().manual_seed(n)).to(torch.int32)
    table = order[:n * pages].clone()
    for k, i in enumerate(bad):
        table[i] = [-1, N, 2 ** 31 - 1, -2 ** 31][k % 4]
    good = [x for x in table.tolist() if 0 <= x < N]
    head, free, ring = N - 5, torch.full((N,), -7, dtype=torch.int32), i32([0, 0])
    free[torch.tensor([(head + i) % N for i in range(9)])] = order[n * pages:]
    free, table = free.cuda(), table.view(n, pages).cuda()
    lens = i32([pages * P - r % P for r in range(n)])
    pg = H.make_page_cfg(P, N, pages)
    H.hybrid_page_release(pg, n, i32(range(n)), n, lens, table, free, i32([head, 9]), ring)
    assert H.hybrid_check(check=False) == (H.HYBRID_ERR_DEVICE if len(bad) else H.HYBRID_OK)
    assert ring.tolist() == [head, 9 + len(good)]
    live = [free.tolist()[(head + i) % N] for i in range(9 + len(good))]
    assert live == order[n * pages:].tolist() + good
    # without entries of that kind, the ring half full: in order, and all of them
    half, again = n * pages // 2, i32([0, 0])
    table = order[:n * pages].view(n, pages).cuda()
    H.hybrid_page_release(pg, n, i32(range(n)), n, lens, table, free, i32([3, half]), again)
    assert H.hybrid_check(check=False) == (H.HYBRID_OK if n * pages <= N - half else H.HYBRID_ERR_DEVICE)
    m = min(n * pages, N - half)
    assert again.tolist() == [3, half + m]
    assert [free.tolist()[(3 + half + i) % N] for i in range(m)] == order[:m].tolist()


# ------------------------------------------------------------------ batches with idle rows

@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("pad", [0, 3])
def test_decoding_after_a_middle_and_the_last_row_are_released(dt, pad):
    """Two blocks, the second for the requests that are left, one of which has fewer tokens than a block."""
    B, n = 4, 5
    cfg = H.make_cfg(64, 64, 4, 2, B, dt)
    pool = PagePool(cfg, n, 200, 600, 16)
    layer = layer_of(pool)

    def block(new, n_tok):
        slots, positions, offsets = pool.append(i32(new), n_tok)
        x = torch.randn(n_tok, 8 * 64, device="cuda").to(dt)
        if max(new) > B:
            return layer.write(x, pool, 0, slots, positions)
        rows = pool.block_rows(offsets, n_tok)
        q = layer.write(x, pool, 0, slots, positions)
        out = layer.attend(q, pool, 0, rows=rows)
        assert torch.equal(out, layer.step(x, pool, 0, slots, positions, rows=rows))     # (writes the same again)
        H.hybrid_check()
        lens, at = pool.lens.tolist(), 0
        for r, m in enumerate(new):
            if m:
                want = R.paged_attention(q[at:at + m][None], pool.k_cache[0], pool.v_cache[0], pool.block_table[r:r + 1], lens[r:r + 1], 0, 0)
                assert_parity(out[at:at + m][None].double().cpu().numpy(), want.cpu().numpy(), dt, f"request {r}", units="out")
            at += m
        assert not bool(out[at:].any())

    block([130, 7, 300, 16, 45], 498)
    block([B] * n, n * B + pad)
    pool.release(i32([2, 4]))
    block([B, B - 1, 0, B, 0], 3 * B - 1 + pad)
    block([B, B, 0, B, 0], n * B)                            # as many as query rows, but not in their places
    block([0, 0, 0, 1, 0], 1 + pad)


# ------------------------------------------------------------------ graphs

def test_a_captured_append_and_release_go_on_from_call_to_call():
    """One append, and one append with one release, captured and replayed among eager calls: lengths, ring and
    tables against the model."""
    P, n, N = 16, 3, 60
    cfg = H.make_cfg(64, 64, 4, 2, 2, F32)
    pool = PagePool(cfg, n, N, 200, P)
    model = R.Pool(P, N, pool.pg.max_pages, range(N), 0, N, [[-1] * pool.pg.max_pages for _ in range(n)])
    lens, held = [0] * n, pool.lens
    new, rows = i32([5, 17, 2]), i32([1])
    pool.append(i32([0, 0, 0]), 24), pool.release(i32([]))
    graphs = []
    for release in (False, True):
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            out = pool.append(new, 24)
            if release:
                pool.release(rows)
        graphs.append((g, out))

    def check(out, n_new):
        nonlocal lens
        H.hybrid_check()
        slots, pos, offs, lens, bad = model.append(lens, n_new, 24)
        assert not bad and [x.tolist() for x in out] == [slots, pos, offs]

    for what in (0, 0, 0, 1, 0, 2, 1, 1, 2, 2, 2, 0):        # the graphs, or an eager append
        if what == 2:
            check(pool.append(i32([1, 0, 4]), 24), [1, 0, 4])
        else:
            graphs[what][0].replay()
            check(graphs[what][1], [5, 17, 2])
        if what == 1:
            model.release([1], lens)
            lens[1] = 0
        assert pool.lens.tolist() == held.tolist() == lens and pool.ring.tolist() == [model.head, model.count]
        assert pool.block_table.tolist() == model.table


@pytest.mark.parametrize("dt", [BF, F32])
def test_graphs_replayed_at_once(dt):
    """Two captured attentions of contexts that are split, replayed on two streams beside eager calls on a third."""
    cfg = H.make_cfg(128, 64, 8, 2, 16, dt)
    pool = filled(cfg, [9000, 20000, 700], 1900, 20000)
    layer = layer_of(pool)
    q = [torch.randn(48, 8, 128, device="cuda").to(dt) for _ in range(3)]
    want = [layer.attend(x, pool, 0) for x in q]
    torch.cuda.synchronize()
    graphs = []
    for x in q[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = layer.attend(x, pool, 0)
        graphs.append((g, out))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for trial in range(30):
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        eager = layer.attend(q[2], pool, 0)
        torch.cuda.synchronize()
        assert torch.equal(eager, want[2]) and all(torch.equal(out, w) for (_, out), w in zip(graphs, want)), trial
    H.hybrid_check()


def test_captured_attention_has_a_workspace_of_its_graph(monkeypatch):
    cfg = H.make_cfg(64, 64, 4, 2, 2, BF)
    pool = filled(cfg, [300, 200, 100], 60, 400)
    layer, q = layer_of(pool), torch.randn(6, 4, 64, device="cuda").to(BF)
    seen, call = [], H.hybrid_paged_attn

    def note(*args, **kw):
        seen.append(args[11].data_ptr())
        return call(*args, **kw)

    monkeypatch.setattr(H, "hybrid_paged_attn", note)
    s, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    layer.attend(q, pool, 0, s)
    torch.cuda.synchronize()
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            layer.attend(q, pool, 0)
    H.hybrid_check()
    assert len(set(seen)) == 3


# ------------------------------------------------------------------ infinities and NaN that queries see

ROWS = [(1, 1), (1, 4), (8, 4), (33, 1), (16, 4), (9, 8), (24, 4), (32, 4), (33, 5)]     # (tokens, heads of a key head)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,G", ROWS)
def test_infinite_and_nan_values_that_queries_see(dt, B, G):
    """One feature of some values is infinite or NaN: that feature of the outputs is what the formula gives (keys are
    small, so that no weight vanishes), whatever the number of rows, and every other output is as without it."""
    from test_gpu_softmax import attn_setup, run_attn
    lens = [300, 128, 1000, 77, 4000]
    s = attn_setup(dt, B, 2 * G, 2, 64, 16, lens, seed=3, k_scale=0.1)
    clean = run_attn(s)
    put = lambda r, j, h, c, x: s["vc"].__setitem__((int(s["table"][r, j // 16]), h, j % 16, c), x)  # noqa: E731
    inf, nan = float("inf"), float("nan")
    put(0, 200, 0, 5, inf), put(0, 299, 1, 63, -inf)         # a last, partial tile; its last key
    put(1, 3, 0, 0, inf), put(1, 100, 0, 0, inf), put(1, 127, 0, 1, -inf)
    put(2, 999, 1, 9, inf), put(2, 500, 1, 9, -inf)          # both signs: NaN
    put(3, 0, 0, 7, nan), put(4, 2000, 0, 30, inf), put(4, 3999, 1, 31, nan)
    got = run_attn(s)
    want = R.paged_attention(s["q"], s["kc"], s["vc"], s["table"], lens, 0, 0)
    odd = ~torch.isfinite(want)
    assert int(odd.sum()) == 8 * B * G
    assert torch.equal(got.double()[odd].nan_to_num(5.0, 1.0, -1.0), want[odd].nan_to_num(5.0, 1.0, -1.0))
    assert torch.equal(got[~odd], clean[~odd])


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,G", ROWS)
def test_infinite_and_nan_keys_and_queries(dt, B, G):
    """A query with NaN gives NaN in its own row alone; a key with an infinity makes each score infinite: NaN where it
    is positive, a weight of zero where it is negative."""
    from test_gpu_softmax import attn_setup, run_attn
    lens = [300, 128, 1000]
    s = attn_setup(dt, B, 2 * G, 2, 64, 16, lens, seed=4)
    s["kc"][int(s["table"][1, 3]), 1, 5, 2] = float("inf")
    s["q"][1, :, G:, 2] = s["q"][1, :, G:, 2].abs() + 1
    s["q"][1, 0, G, 2] *= -1
    s["q"][2, B - 1, 0, 11] = float("nan")
    got = run_attn(s)
    want = R.paged_attention(s["q"], s["kc"], s["vc"], s["table"], lens, 0, 0)
    odd = want.isnan()
    assert int(odd.sum()) == 64 * (B * G - 1 + 1) and torch.equal(got.isnan(), odd)
    assert_parity(got.double().nan_to_num(0.0).cpu().numpy(), want.nan_to_num(0.0).cpu().numpy(), dt, "the rest", units="out")
