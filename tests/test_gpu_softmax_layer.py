"""The pool and the layer of the softmax layers as a serving loop uses them: streams, batches with idle
rows, graphs, and infinities in the cache."""
import pytest
import torch

from paper_2608_06628_gb300 import hybrid as H
from paper_2608_06628_gb300.page_pool import PagePool

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
