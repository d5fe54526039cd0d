"""The softmax-layer operators on the GPU against plain implementations in 64 bits.

Bounds, from the arithmetic (eps32 = 2^-24, bf16 rounding: half an ulp <= 2^-8 |value|):
  rotation   float32: mean square, rsqrt, weight, angle and two products are each a few eps32 of the
             row's largest entry: 32 eps32 = 2e-6 of it; bf16 adds the output's rounding.
  gradient   dx: the same operations on r u, whose terms cancel: 64 eps32 = 4e-6 of the largest |r u|
             term of the row; dw = sum dn xh: float32 sums of up to 50 terms in a row, 50 eps32 of
             sum |terms|, and in every term the rotation's error of dn (32 eps32 of the row's largest
             dy, however small the rotated dn is by cancellation) times |xh|.
  attention  the bounds that the block-hybrid step is held to (gpu_harness.TOL): float32 rel-L2 1e-5 and
             max-abs 1e-4; bf16 rel-L2 1e-2 of every (request, head): probabilities and outputs are
             rounded to bf16, 2^-9 of the norm each at most.
Whole numbers are equal.
"""
import math
import random

import numpy as np
import pytest
import torch

import softmax_reference as R
from gpu_harness import assert_parity
from paper_2608_06628_gb300 import hybrid as H

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_06628_gb300 import build
    build.build()
    torch.cuda.set_device(0)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------ pages

def make_pool(rng, P, lens, n_pages, max_pages):
    ids = list(range(n_pages))
    rng.shuffle(ids)
    table = [[-1] * max_pages for _ in lens]
    for r, x in enumerate(lens):
        for j in range(-(-max(x, 0) // P)):
            if j < max_pages:
                table[r][j] = ids.pop()
    head = rng.randrange(n_pages)
    free = [-5] * n_pages
    for i, p in enumerate(ids):
        free[(head + i) % n_pages] = p
    return R.Pool(P, n_pages, max_pages, free, head, len(ids), table)


def append_gpu(pool, lens, new, n_slots, optional=True):
    n = len(lens)
    pg = H.make_page_cfg(pool.P, pool.N, pool.max_pages)
    t = dict(table=i32(pool.table) if n else None, slots=torch.full((max(n_slots, 1),), 77, dtype=torch.int32, device="cuda"),
             pos=torch.full((max(n_slots, 1),), 77, dtype=torch.int32, device="cuda") if optional else None,
             offs=i32([77] * (n + 1)) if optional else None, out=i32([77] * max(n, 1)), ring=i32([7, 7]))
    H.hybrid_page_append(pg, n, i32(lens or [0]), i32(new or [0]), i32(pool.free), i32([pool.head, pool.count]), t["table"],
                         t["slots"], t["pos"], n_slots, t["offs"], t["out"], t["ring"])
    return t


def check_append(pool, lens, new, n_slots):
    t = append_gpu(pool, lens, new, n_slots)
    st = H.hybrid_check(check=False)
    slots, pos, offs, out, bad = pool.append(lens, new, n_slots)
    assert st == (H.HYBRID_ERR_DEVICE if bad else H.HYBRID_OK)
    assert t["slots"].tolist()[:n_slots] == slots and t["pos"].tolist()[:n_slots] == pos
    assert t["offs"].tolist() == offs
    assert t["ring"].tolist() == [pool.head, pool.count]
    if lens:
        assert t["out"].tolist() == out and t["table"].tolist() == pool.table
    return out


@pytest.mark.parametrize("n,P,len_max,new_max,spare", [
    (1, 16, 0, 1, 0), (1, 128, 1, 300, 3), (7, 16, 100, 40, 0), (64, 32, 8192, 32, 5), (333, 64, 50, 700, 9),
    (2500, 16, 40, 33, 1), (1025, 128, 3, 0, 4),
])
def test_append_and_release(n, P, len_max, new_max, spare):
    rng = random.Random(n * 1000 + P)
    for trial in range(3):
        lens = [rng.choice([0, P, rng.randint(0, len_max)]) if len_max >= P else rng.randint(0, len_max) for _ in range(n)]
        new = [rng.randint(0, new_max) for _ in range(n)]
        max_pages = max(1, -(-max(x + y for x, y in zip(lens, new)) // P))
        need = sum(-(-(x + y) // P) for x, y in zip(lens, new))
        pool = make_pool(rng, P, lens, need + spare + 1, max_pages)
        n_slots = sum(new) + (0 if trial == 0 else rng.randint(0, 600))
        out = check_append(pool, lens, new, n_slots)
        rows = rng.sample(range(n), rng.randint(0, n))
        free = i32(pool.free)
        ring = i32([5, 5])
        H.hybrid_page_release(H.make_page_cfg(P, pool.N, max_pages), n, i32(rows or [0]), len(rows), i32(out), i32(pool.table),
                              free, i32([pool.head, pool.count]), ring)
        H.hybrid_check()
        pool.release(rows, out)
        assert ring.tolist() == [pool.head, pool.count]
        # the live part of the ring (the rest is unspecified)
        live = lambda f: [f[(pool.head + i) % pool.N] for i in range(pool.count)]  # noqa: E731
        assert live(free.tolist()) == live(pool.free)


def test_append_refuses_what_does_not_fit():
    """Too few pages, a row longer than the table, negative numbers, too few slots: the requests concerned
    stay as they are, the others are served, and the check reports it."""
    rng = random.Random(3)
    P = 16
    lens, new = [16, 5, 0, 31, 40], [16, 11, 33, 1, 8]        # need 1, 0, 3, 0, 0 pages
    pool = make_pool(rng, P, lens, 1 + sum(-(-x // P) for x in lens), 8)
    assert pool.count == 1
    check_append(pool, lens, new, 80)
    for lens, new, n_slots, max_pages in [([-1, 3, 7], [4, 4, 4], 20, 4), ([3, 3, 3], [4, -9, 4], 20, 4),
                                          ([3, 60, 3], [4, 5, 4], 20, 4), ([3, 3, 3], [4, 5, 4], 10, 4),
                                          ([3, 2147483647, 0], [4, 2147483647, 16], 40, 4),
                                          ([3, 5, 0], [4, 2147483647, 16], 40, 4)]:
        pool = make_pool(rng, P, [min(max(x, 0), 64) for x in lens], 40, max_pages)
        check_append(pool, lens, new, n_slots)
    # a ring out of range serves nothing that needs a page, and stays
    pool = make_pool(rng, P, [3, 4], 10, 4)
    t = append_gpu(R.Pool(P, 10, 4, pool.free, 10, 3, pool.table), [3, 4], [1, 20], 21)
    assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
    assert t["ring"].tolist() == [10, 3] and t["out"].tolist() == [4, 4]
    # page numbers out of range give slot -1
    bad = R.Pool(P, 10, 4, [99] * 10, 0, 10, pool.table)
    t = append_gpu(bad, [3, 4], [1, 20], 21)
    assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
    assert t["slots"].tolist()[0] == pool.table[0][0] * P + 3 and t["slots"].tolist()[13:] == [-1] * 8


def test_append_without_optional_outputs_and_without_requests():
    rng = random.Random(4)
    pool = make_pool(rng, 32, [5, 40], 9, 3)
    t = append_gpu(pool, [5, 40], [30, 2], 40, optional=False)
    H.hybrid_check()
    assert t["slots"].tolist() == pool.append([5, 40], [30, 2], 40)[0]
    pool = make_pool(rng, 32, [], 9, 3)
    t = append_gpu(pool, [], [], 5)
    H.hybrid_check()
    assert t["slots"].tolist() == [-1] * 5 and t["offs"].tolist() == [0] and t["ring"].tolist() == [pool.head, pool.count]


def test_release_reports_bad_rows_and_a_full_ring():
    rng = random.Random(5)
    pool = make_pool(rng, 16, [40, 10], 6, 3)
    pg = H.make_page_cfg(16, 6, 3)
    for rows, lens in [([2], [40, 10]), ([-1, 0], [40, 10]), ([0], [-3, 10]), ([0], [1000, 10])]:
        free, ring = i32(pool.free), i32([0, 0])
        H.hybrid_page_release(pg, 2, i32(rows), len(rows), i32(lens), i32(pool.table), free, i32([pool.head, pool.count]), ring)
        assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
        assert ring.tolist() == [pool.head, pool.count + (3 if rows == [-1, 0] else 0)]
    free, ring = i32([9] * 6), i32([0, 0])
    H.hybrid_page_release(pg, 2, i32([0, 1]), 2, i32([40, 10]), i32(pool.table), free, i32([1, 4]), ring)   # room for 2 of 4
    assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
    assert ring.tolist() == [1, 6] and free.tolist() == [pool.table[0][1], 9, 9, 9, 9, pool.table[0][0]]


# ------------------------------------------------------------------ norm and rotation

def rope_setup(T, Hq, Hkv, d, rot, dt, inter=False, norm=True, kind="none", factor=1.0, seed=0, max_pos=100000):
    g = gen(seed)
    qkv = torch.randn(T, (Hq + 2 * Hkv) * d + 16, generator=g, device="cuda").to(dt)    # 16 elements of something else
    q, k, v = (qkv[:, a:b] for a, b in ((0, Hq * d), (Hq * d, (Hq + Hkv) * d), ((Hq + Hkv) * d, (Hq + 2 * Hkv) * d)))
    w = (1 + 0.3 * torch.randn(2, d, generator=g, device="cuda")).to(dt)
    kinds = {"none": H.HYBRID_ROPE_NONE, "linear": H.HYBRID_ROPE_LINEAR, "ntk": H.HYBRID_ROPE_NTK, "yarn": H.HYBRID_ROPE_YARN}
    rope, freqs = H.make_rope(rot, inter, eps=EPS, kind=kinds[kind], factor=factor)
    t, scale = R.turns(rot, kind, factor=factor)
    assert abs(rope.scale - scale) <= 1e-7 * scale
    pos = torch.randint(0, max_pos, (T,), generator=g, device="cuda", dtype=torch.int32)
    return dict(cfg=H.make_cfg(d, 64, Hq, Hkv, 1, dt), rope=rope, freqs=freqs, q=q.view(T, Hq, d), k=k.view(T, Hkv, d),
                v=v.view(T, Hkv, d), stride=qkv.stride(0), wq=w[0] if norm else None, wk=w[1] if norm else None, pos=pos, t=t,
                scale=scale, inter=inter, dt=dt, T=T, Hq=Hq, Hkv=Hkv, d=d)


def want_rope(s, x, w):
    return R.norm_rotate(x.double(), None if w is None else w.double(), s["pos"], s["t"], s["scale"], s["inter"], EPS)


def close_rows(got, want, dt, what, rel=2e-6):
    got, tol = got.double(), rel * want.abs().amax(-1, keepdim=True)
    if dt == BF:
        tol = tol + want.abs() * 2.0 ** -8
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((got - want).abs().max()):.3e}"


def run_rope(s, stream=None):
    qo = torch.empty(s["T"], s["Hq"], s["d"], dtype=s["dt"], device="cuda")
    ko = torch.empty(s["T"], s["Hkv"], s["d"], dtype=s["dt"], device="cuda")
    H.hybrid_qk_norm_rope(s["cfg"], s["rope"], s["q"], s["stride"], s["k"], s["stride"], s["T"], s["wq"], s["wk"], s["pos"],
                          s["freqs"], qo, ko, stream=stream)
    return qo, ko


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,inter,norm,kind,factor", [
    (1, 1, 1, 64, 64, False, True, "none", 1.0), (3, 16, 4, 128, 128, False, True, "none", 1.0),
    (65, 16, 4, 128, 128, True, True, "yarn", 8.0), (257, 5, 5, 64, 16, False, True, "linear", 4.0),
    (129, 6, 2, 128, 96, False, False, "ntk", 2.0), (40, 7, 1, 128, 80, True, False, "none", 1.0),
    (33, 3, 3, 64, 48, True, True, "ntk", 16.0), (2049, 8, 8, 64, 64, False, True, "yarn", 4.0),
    (5000, 16, 4, 128, 0, False, True, "none", 1.0), (20, 256, 1, 128, 112, False, True, "none", 1.0),
])
def test_norm_and_rotation(dt, T, Hq, Hkv, d, rot, inter, norm, kind, factor):
    s = rope_setup(T, Hq, Hkv, d, rot, dt, inter, norm, kind, factor, seed=T + rot)
    qo, ko = run_rope(s)
    H.hybrid_check()
    close_rows(qo, want_rope(s, s["q"], s["wq"]), dt, "q")
    close_rows(ko, want_rope(s, s["k"], s["wk"]), dt, "k")


def test_rotation_at_every_position_an_int_holds():
    """The angle is exact in integers: far and negative positions are as good as near ones."""
    T, d = 64, 128
    s = rope_setup(T, 2, 2, d, d, F32, norm=False)
    pos = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 123456789, -987654321] * 8
    s["pos"] = i32(pos)
    f = [int(x) & (2 ** 64 - 1) for x in s["freqs"].tolist()]
    # the reference's fraction of a turn, in Python's integers from the same frequencies
    frac = torch.tensor([[((p * x) & (2 ** 64 - 1)) / 2.0 ** 64 for x in f] for p in pos], dtype=torch.float64, device="cuda")
    c, sn = torch.cos(2 * math.pi * frac)[:, None], torch.sin(2 * math.pi * frac)[:, None]
    qo, ko = run_rope(s)
    for got, x in ((qo, s["q"].double()), (ko, s["k"].double())):
        a, b = x[..., :64], x[..., 64:]
        close_rows(got, torch.cat([a * c - b * sn, b * c + a * sn], -1), F32, "far positions")


def test_norm_in_place_tiny_rows_and_unrotated_infinities():
    s = rope_setup(50, 4, 2, 64, 32, BF, seed=9)
    q, k = s["q"].clone(), s["k"].clone()                    # dense
    q[3] = 0                                                 # rsqrt(eps), not a division by zero
    q[4] *= 1e-20
    want_q, want_k = want_rope(s, q, s["wq"]), want_rope(s, k, s["wk"])
    H.hybrid_qk_norm_rope(s["cfg"], s["rope"], q, 4 * 64, k, 2 * 64, 50, s["wq"], s["wk"], s["pos"], s["freqs"], q, k)
    close_rows(q, want_q, BF, "in place q")
    close_rows(k, want_k, BF, "in place k")
    assert bool((q[3] == 0).all())
    q = s["q"].clone()
    q[..., 40] = math.inf                                    # beyond rot_dim, no norm: passes through
    out, ko = torch.empty_like(q), torch.empty_like(k)
    H.hybrid_qk_norm_rope(s["cfg"], s["rope"], q, 4 * 64, k, 2 * 64, 50, None, None, s["pos"], s["freqs"], out, ko)
    assert bool((out[..., 40] == math.inf).all()) and bool(torch.isfinite(out[..., :32]).all())


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,d,P", [(1, 1, 1, 64, 16), (64, 16, 4, 128, 32), (700, 6, 3, 64, 128), (2048, 16, 4, 128, 16)])
def test_cache_writes(dt, T, Hq, Hkv, d, P):
    s = rope_setup(T, Hq, Hkv, d, d, dt, seed=T)
    n_pages = -(-T // P) + 2
    slots = torch.randperm(n_pages * P, generator=gen(1), device="cuda")[:T].to(torch.int32)
    if T > 1:
        slots[::7] = -1
    kc = torch.full((n_pages, Hkv, P, d), 7.0, dtype=dt, device="cuda")
    vc = torch.full((n_pages, Hkv, P, d), 7.0, dtype=dt, device="cuda")
    qo, ko = run_rope(s)
    q2 = torch.empty_like(qo)
    H.hybrid_qk_norm_rope_cache(s["cfg"], s["rope"], H.make_page_cfg(P, n_pages, 1), s["q"], s["stride"], s["k"], s["stride"],
                                s["v"], s["stride"], T, s["wq"], s["wk"], s["pos"], s["freqs"], slots, q2, kc, vc)
    H.hybrid_check()
    assert torch.equal(q2, qo)
    wk, wv = torch.full_like(kc, 7.0), torch.full_like(vc, 7.0)
    live = slots >= 0
    sl = slots[live].long()
    wk[sl // P, :, sl % P] = ko[live]
    wv[sl // P, :, sl % P] = s["v"][live]
    assert torch.equal(kc, wk) and torch.equal(vc, wv)
    # beyond the pool: nothing written, reported
    slots[0] = n_pages * P
    slots[T // 2] = 2 ** 31 - 1
    kc.fill_(7.0)
    H.hybrid_qk_norm_rope_cache(s["cfg"], s["rope"], H.make_page_cfg(P, n_pages, 1), s["q"], s["stride"], s["k"], s["stride"],
                                s["v"], s["stride"], T, s["wq"], s["wk"], s["pos"], s["freqs"], slots, q2, kc, vc)
    assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
    assert H.hybrid_check(check=False) == H.HYBRID_OK
    assert torch.equal(q2, qo)


def run_backward(s, dqo, dko):
    T, Hq, Hkv, d = s["T"], s["Hq"], s["Hkv"], s["d"]
    wide = torch.full((T, s["stride"]), 5.0, dtype=s["dt"], device="cuda")
    dq, dk = wide[:, :Hq * d].view(T, Hq, d), wide[:, Hq * d:(Hq + Hkv) * d].view(T, Hkv, d)
    norm = s["wq"] is not None
    dw = torch.full((2, d), 9.0, dtype=F32, device="cuda")
    nb = H.hybrid_qk_norm_rope_workspace_bytes(s["cfg"], T)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")      # NaN patterns
    H.hybrid_qk_norm_rope_backward(s["cfg"], s["rope"], s["q"], s["stride"], s["k"], s["stride"], dqo, dko, T, s["wq"],
                                   s["wk"], s["pos"], s["freqs"], ws, nb, dq, dk, dw[0] if norm else None,
                                   dw[1] if norm else None)
    H.hybrid_check()
    assert bool((wide[:, (Hq + Hkv) * d:] == 5.0).all())               # the rest of the rows is left alone
    return dq, dk, dw


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,inter,norm", [
    (1, 1, 1, 64, 64, False, True), (5, 16, 4, 128, 128, False, True), (333, 6, 3, 64, 48, True, True),
    (2500, 16, 4, 128, 96, False, True), (77, 5, 1, 128, 128, True, False), (9, 256, 1, 64, 0, False, True),
    (12000, 3, 3, 64, 64, False, True),
])
def test_gradient(dt, T, Hq, Hkv, d, rot, inter, norm):
    s = rope_setup(T, Hq, Hkv, d, rot, dt, inter, norm, "yarn" if rot else "none", 4.0 if rot else 1.0, seed=T)
    g = gen(T + 1)
    dqo, dko = (torch.randn(T, h, d, generator=g, device="cuda").to(dt) for h in (Hq, Hkv))
    dq, dk, dw = run_backward(s, dqo, dko)
    for name, x, w, dy, dx, got_w in (("q", s["q"], s["wq"], dqo, dq, dw[0]), ("k", s["k"], s["wk"], dko, dk, dw[1])):
        w64 = None if w is None else w.double()
        want, want_w, size = R.norm_rotate_grad(x.double(), w64, dy.double(), s["pos"], s["t"], s["scale"], inter, EPS)
        # the terms that cancel in dx are as large as r u
        xd = x.double()
        r = ((xd * xd).mean(-1, keepdim=True) + EPS).rsqrt() if w is not None else 1.0
        u = R.norm_rotate(dy.double(), None, -s["pos"].long(), s["t"], s["scale"], inter, EPS)
        big = (r * u * (w64 if w64 is not None else 1.0)).abs().amax(-1, keepdim=True) * (1 + (dt == F32))
        tol = 4e-6 * big + (want.abs() * 2.0 ** -8 if dt == BF else 0)
        assert not bool(((dx.double() - want).abs() > tol).any()), f"d{name}"
        if w is not None:
            # up to ceil(rows / (608 blocks * 8 warps)) terms in a lane's sum, then 13 more additions
            terms = max(50, T * (Hq + Hkv) // 4864 + 13)
            dn_err = 2e-6 * s["scale"] * dy.double().abs().amax(-1, keepdim=True)
            tol = terms * 2.0 ** -24 * size + (dn_err * (xd * r).abs()).sum((0, 1))
            assert not bool(((got_w.double() - want_w).abs() > tol).any()), f"dw{name}"
    again = run_backward(s, dqo, dko)
    assert torch.equal(dq, again[0]) and torch.equal(dk, again[1]) and torch.equal(dw, again[2])


def test_gradient_against_differences():
    """Central differences of the 64-bit forward pass along random directions: error of order h^2 = 1e-8,
    and 1e-9 from cancellation at h = 1e-4; the float32 gradient adds about 1e-6: 1e-5 of the scale."""
    s = rope_setup(37, 4, 2, 64, 48, F32, True, True, "yarn", 4.0, seed=3)
    g = gen(8)
    dqo, dko = (torch.randn(37, h, 64, generator=g, device="cuda") for h in (4, 2))
    dq, dk, dw = run_backward(s, dqo, dko)
    h = 1e-4
    for x, w, dy, dx, got_w in ((s["q"], s["wq"], dqo, dq, dw[0]), (s["k"], s["wk"], dko, dk, dw[1])):
        x, w, dy = x.double(), w.double(), dy.double()
        loss = lambda x, w: (dy * want_rope(s, x, w)).sum()  # noqa: E731, B023
        for trial in range(4):
            ex = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
            ew = torch.randn(w.shape, generator=g, device="cuda", dtype=torch.float64)
            for e, at, got in ((ex, "x", (dx.double() * ex).sum()), (ew, "w", (got_w.double() * ew).sum())):
                up = loss(x + h * e, w) if at == "x" else loss(x, w + h * e)
                down = loss(x - h * e, w) if at == "x" else loss(x, w - h * e)
                size = float(((dx.double() * ex).abs() if at == "x" else (got_w.double() * ew).abs()).sum())
                assert abs(float(got) - float((up - down) / (2 * h))) <= 1e-5 * size, at


def test_no_tokens():
    s = rope_setup(1, 2, 2, 64, 64, F32)
    s["T"] = 0
    dw = torch.full((2, 64), 9.0, device="cuda")
    nb = H.hybrid_qk_norm_rope_workspace_bytes(s["cfg"], 0)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    H.hybrid_qk_norm_rope_backward(s["cfg"], s["rope"], None, 0, None, 0, None, None, 0, s["wq"], s["wk"], None, None, ws, nb,
                                   None, None, dw[0], dw[1])
    H.hybrid_qk_norm_rope(s["cfg"], s["rope"], None, 0, None, 0, 0, s["wq"], s["wk"], None, None, None, None)
    H.hybrid_check()
    assert bool((dw == 0).all())


# ------------------------------------------------------------------ attention

def attn_setup(dt, B, Hq, Hkv, d, P, lens, window=0, sink=0, seed=0, k_scale=1.0, poison=True):
    """A cache in which every place that no query sees holds NaN, pages that hold no visible key are not in
    the pool at all, and their table entries are out of range."""
    g, rng = gen(seed), random.Random(seed)
    n = len(lens)
    max_pages = max(1, -(-max(lens) // P)) + 1
    seen = [R.visible(x, window, sink) for x in lens]
    pages = [sorted({j // P for j in v}) for v in seen]
    n_pages = sum(map(len, pages)) + 2
    ids = list(range(n_pages))
    rng.shuffle(ids)
    table = torch.full((n, max_pages), -77 if seed % 2 else 2 ** 30, dtype=torch.int32)
    fill = math.nan if poison else 0.0
    kc = torch.full((n_pages, Hkv, P, d), fill, dtype=dt, device="cuda")
    vc = torch.full((n_pages, Hkv, P, d), fill, dtype=dt, device="cuda")
    for r in range(n):
        for j in pages[r]:
            table[r, j] = ids.pop()
        if seen[r]:
            j = torch.tensor(seen[r])
            page, at = table[r][j // P].long().cuda(), (j % P).cuda()
            kc[page, :, at] = (torch.randn(len(j), Hkv, d, generator=g, device="cuda") * k_scale).to(dt)
            vc[page, :, at] = torch.randn(len(j), Hkv, d, generator=g, device="cuda").to(dt)
    return dict(cfg=H.make_cfg(d, 64, Hq, Hkv, B, dt), pg=H.make_page_cfg(P, n_pages, max_pages), kc=kc, vc=vc,
                q=torch.randn(n, B, Hq, d, generator=g, device="cuda").to(dt), table=table.cuda(), lens=i32(lens), n=n,
                window=window, sink=sink, dt=dt)


def run_attn(s, stream=None):
    o = torch.full_like(s["q"], 3.0)
    nb = H.hybrid_paged_attn_workspace_bytes(s["cfg"], s["pg"], s["n"])
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    H.hybrid_paged_attn(s["cfg"], s["pg"], s["q"], s["kc"], s["vc"], s["table"], s["lens"], s["n"], s["window"], s["sink"], o,
                        ws, nb, stream=stream)
    H.hybrid_check(stream=stream)
    return o


def check_attn(s, what=""):
    o = run_attn(s)
    want = R.paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["lens"].tolist(), s["window"], s["sink"])
    got, want = o.double().cpu().numpy(), want.cpu().numpy()
    assert_parity(got, want, s["dt"], what, units="out")
    for r, x in enumerate(s["lens"].tolist()):
        if not R.visible(x, s["window"], s["sink"]):
            assert not np.any(got[r]), "zeros without a visible key"
    return o


EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 1000]


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,Hq,Hkv,d,P", [
    (1, 16, 4, 128, 16), (1, 1, 1, 64, 128), (32, 16, 4, 128, 32), (16, 2, 2, 64, 64), (33, 6, 2, 128, 16), (128, 4, 4, 64, 32),
    (1, 32, 1, 128, 64), (5, 35, 5, 64, 16), (3, 160, 1, 128, 16), (2, 256, 1, 64, 128), (64, 16, 4, 128, 128),
])
def test_attention_edges_of_pages_and_tiles(dt, B, Hq, Hkv, d, P):
    check_attn(attn_setup(dt, B, Hq, Hkv, d, P, EDGES, seed=B + Hq), f"B{B} Hq{Hq} Hkv{Hkv} d{d} P{P}")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (16, 4), (100, 0), (128, 128), (129, 33), (1000, 130), (257, 500),
                                         (5, 100000), (2147483647, 7)])
def test_attention_window_and_first_tokens(dt, window, sink):
    lens = [0, 1, 5, 16, 100, 129, 140, 256, 260, 385, 512, 777, 1500, 4000]
    for B, Hq, Hkv, d, P in ((1, 8, 2, 128, 16), (32, 4, 1, 64, 64)):
        check_attn(attn_setup(dt, B, Hq, Hkv, d, P, lens, window, sink, seed=window % 97 + sink % 31), f"window {window} sink {sink}")


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_long_and_split(dt):
    """Requests split over many blocks beside short ones."""
    check_attn(attn_setup(dt, 1, 8, 2, 128, 64, [40001, 3, 17000, 0, 128]), "long, one token")
    check_attn(attn_setup(dt, 32, 4, 1, 128, 32, [20011, 1, 9000]), "long, block")
    check_attn(attn_setup(dt, 1, 1, 1, 64, 16, [9999]), "one head")


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_many_requests(dt):
    rng = random.Random(1)
    lens = [rng.choice([0, 1, 16, rng.randint(0, 200)]) for _ in range(3000)]
    check_attn(attn_setup(dt, 1, 4, 2, 64, 16, lens), "3000 requests")
    check_attn(attn_setup(dt, 1, 4, 2, 64, 16, [0] * 300 + [5] + [0] * 300), "mostly empty")
    check_attn(attn_setup(dt, 4, 4, 2, 64, 16, [0] * 40), "all empty")


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_large_scores(dt):
    """Keys eight times as large: one key takes nearly all of the softmax, and the running maximum moves."""
    check_attn(attn_setup(dt, 32, 16, 4, 128, 32, [700, 33, 4000], k_scale=8.0), "k x 8")
    s = attn_setup(dt, 4, 8, 2, 64, 16, [3000])
    # scores that rise along the cache, so that every tile raises the maximum
    ramp = torch.linspace(0.0, 6.0, 3000, device="cuda")
    page, at = s["table"][0][torch.arange(3000) // 16].long(), torch.arange(3000, device="cuda") % 16
    s["kc"][page, :, at] = (s["kc"][page, :, at].float() * 0.1 + ramp[:, None, None]).to(dt)
    s["q"] = s["q"].abs()
    check_attn(s, "rising scores")


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_same_bits_and_another_stream(dt):
    s = attn_setup(dt, 8, 8, 2, 128, 16, [5000, 77, 1234])
    a = run_attn(s)
    b = run_attn(s, torch.cuda.Stream())
    assert torch.equal(a, b)


def test_attention_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements, whose far pages are used."""
    P, n_pages, Hkv, d = 128, 140000, 1, 128
    assert n_pages * P * d > 2 ** 31
    kc = torch.empty(n_pages, Hkv, P, d, dtype=BF, device="cuda")
    vc = torch.empty(n_pages, Hkv, P, d, dtype=BF, device="cuda")
    s = attn_setup(BF, 1, 4, 1, d, P, [3000, 129])
    for r in range(2):
        for j in range(-(-[3000, 129][r] // P)):
            to, frm = n_pages - 1 - 50 * r - j, int(s["table"][r, j])
            kc[to], vc[to] = s["kc"][frm], s["vc"][frm]
            s["table"][r, j] = to
    s.update(kc=kc, vc=vc, pg=H.make_page_cfg(P, n_pages, s["pg"].max_pages))
    check_attn(s, "far pages")
    # and cache writes there
    r = rope_setup(3, 4, 1, d, d, BF)
    slots = i32([n_pages * P - 1, n_pages * P - 500, 5])
    qo, ko = run_rope(r)
    H.hybrid_qk_norm_rope_cache(r["cfg"], r["rope"], s["pg"], r["q"], r["stride"], r["k"], r["stride"], r["v"], r["stride"], 3,
                                r["wq"], r["wk"], r["pos"], r["freqs"], slots, torch.empty_like(qo), kc, vc)
    H.hybrid_check()
    sl = slots.long()
    assert torch.equal(kc[sl // P, :, sl % P], ko) and torch.equal(vc[sl // P, :, sl % P], r["v"])


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_reports_bad_pages_and_lengths(dt):
    """A page or length out of range is reported; the other requests are right, and nothing out of bounds is read."""
    for bad_page in (-1, 10 ** 6):
        s = attn_setup(dt, 2, 4, 2, 64, 16, [300, 200, 100], poison=False)
        want = R.paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["lens"].tolist(), 0, 0)
        s["table"][1, 3] = bad_page
        o = torch.empty_like(s["q"])
        nb = H.hybrid_paged_attn_workspace_bytes(s["cfg"], s["pg"], 3)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        H.hybrid_paged_attn(s["cfg"], s["pg"], s["q"], s["kc"], s["vc"], s["table"], s["lens"], 3, 0, 0, o, ws, nb)
        assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
        for r in (0, 2):
            assert_parity(o[r:r + 1].double().cpu().numpy(), want[r:r + 1].cpu().numpy(), dt, "beside a bad page", units="out")
    for bad_len in (-5, 2 ** 31 - 1):
        s = attn_setup(dt, 2, 4, 2, 64, 16, [300, 200, 100], poison=False)
        s["table"].clamp_(0, s["pg"].n_pages - 1)
        want = R.paged_attention(s["q"], s["kc"], s["vc"], s["table"], s["lens"].tolist(), 0, 0)
        s["lens"][0] = bad_len
        o = torch.empty_like(s["q"])
        H.hybrid_paged_attn(s["cfg"], s["pg"], s["q"], s["kc"], s["vc"], s["table"], s["lens"], 3, 0, 0, o, ws, nb)
        assert H.hybrid_check(check=False) == H.HYBRID_ERR_DEVICE
        assert_parity(o[1:].double().cpu().numpy(), want[1:].cpu().numpy(), dt, "beside a bad length", units="out")
    assert H.hybrid_check(check=False) == H.HYBRID_OK


# ------------------------------------------------------------------ together

def test_pool_over_many_blocks():
    """Requests that grow block by block, finish and give way to others: the pool against the model."""
    from paper_2608_06628_gb300.page_pool import PagePool
    rng = random.Random(7)
    n, P, B = 9, 16, 5
    pool = PagePool(H.make_cfg(64, 64, 2, 1, B, F32), n, 60, 200, P)
    model = R.Pool(P, 60, pool.pg.max_pages, range(60), 0, 60, [[-1] * pool.pg.max_pages for _ in range(n)])
    lens = [0] * n
    for step in range(40):
        new = [B if x else rng.choice([0, 0, 1, 30, 90]) for x in lens]
        room = sum(new) + rng.randint(0, 9)
        slots, pos, offs = pool.append(i32(new), room)
        st = H.hybrid_check(check=False)
        ws, wp, wo, lens, bad = model.append(lens, new, room)
        assert st == (H.HYBRID_ERR_DEVICE if bad else H.HYBRID_OK)
        assert (slots.tolist(), pos.tolist(), offs.tolist()) == (ws, wp, wo)
        rows = [r for r in range(n) if lens[r] > 100 or (lens[r] and rng.random() < 0.1)]
        if rows:
            pool.release(i32(rows))
            H.hybrid_check()
            model.release(rows, lens)
            lens = [0 if r in rows else x for r, x in enumerate(lens)]
        assert pool.lens.tolist() == lens and pool.ring.tolist() == [model.head, model.count]
        held = sum(-(-x // P) for x in lens)
        assert held + model.count == 60


def test_example_runs_the_operators_together(capsys):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_stack_decode.py")
    spec = importlib.util.spec_from_file_location("hybrid_stack_decode", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    us, err = m.main(["--requests", "5", "--prompt-max", "300", "--blocks", "2", "--steps", "2"])
    assert us > 0 and err <= 1e-2


@pytest.mark.parametrize("dt", [BF, F32])
def test_decoding_in_a_graph(dt):
    """Cache write and attention captured once and replayed on other inputs, one token per request."""
    n, Hq, Hkv, d, P = 6, 8, 2, 64, 16
    s = attn_setup(dt, 1, Hq, Hkv, d, P, [40, 1, 129, 500, 16, 33], poison=False)
    r = rope_setup(n, Hq, Hkv, d, d, dt, seed=2)
    lens = s["lens"].tolist()
    slots = i32([int(s["table"][i, (x - 1) // P]) * P + (x - 1) % P for i, x in enumerate(lens)])
    q, o = torch.empty(n, Hq, d, dtype=dt, device="cuda"), torch.empty(n, 1, Hq, d, dtype=dt, device="cuda")
    nb = H.hybrid_paged_attn_workspace_bytes(s["cfg"], s["pg"], n)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")

    def step():
        H.hybrid_qk_norm_rope_cache(r["cfg"], r["rope"], s["pg"], r["q"], r["stride"], r["k"], r["stride"], r["v"],
                                    r["stride"], n, r["wq"], r["wk"], r["pos"], r["freqs"], slots, q, s["kc"], s["vc"])
        H.hybrid_paged_attn(s["cfg"], s["pg"], q, s["kc"], s["vc"], s["table"], s["lens"], n, 0, 0, o, ws, nb)

    step()
    H.hybrid_check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in (11, 12):
        for x in ("q", "k", "v"):
            r[x].copy_(torch.randn(r[x].shape, generator=gen(seed), device="cuda"))
        g.replay()
        H.hybrid_check()
        close_rows(q, want_rope(r, r["q"], r["wq"]), dt, "q")
        want = R.paged_attention(q[:, None], s["kc"], s["vc"], s["table"], lens, 0, 0)
        assert_parity(o.double().cpu().numpy(), want.cpu().numpy(), dt, "replay", units="out")


@pytest.mark.parametrize("dt", [BF, F32])
def test_attention_row_tiles_of_many_requests(dt):
    """More query rows than one tile holds, with few and with many requests (which share out their work differently)."""
    rng = random.Random(2)
    for n in (3, 128, 129, 400):
        lens = [rng.choice([0, 1, 127, 128, rng.randint(0, 400)]) for _ in range(n)]
        check_attn(attn_setup(dt, 40, 14, 2, 64, 32, lens, seed=n), f"{n} requests, 280 rows")
    check_attn(attn_setup(dt, 128, 8, 1, 128, 16, [3000, 0, 50], 700, 30), "1024 rows, window")


def test_attention_float32_offsets_beyond_32_bits():
    """A float32 cache of more than 2^31 elements, whose far pages are used, with few and with many rows."""
    P, n_pages, d = 128, 140000, 128
    assert n_pages * P * d > 2 ** 31
    kc = torch.empty(n_pages, 1, P, d, device="cuda")
    vc = torch.empty(n_pages, 1, P, d, device="cuda")
    for B in (1, 24):
        s = attn_setup(F32, B, 4, 1, d, P, [3000, 129])
        for r in range(2):
            for j in range(-(-[3000, 129][r] // P)):
                to, frm = n_pages - 1 - 50 * r - j, int(s["table"][r, j])
                kc[to], vc[to] = s["kc"][frm], s["vc"][frm]
                s["table"][r, j] = to
        s.update(kc=kc, vc=vc, pg=H.make_page_cfg(P, n_pages, s["pg"].max_pages))
        check_attn(s, f"far pages, {B} tokens")


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("max_len", [16, 128, 144])
def test_attention_of_contexts_that_fit_a_tile(dt, max_len):
    """The table's width bounds the contexts to one tile (nothing to join) or just above it."""
    lens = [0, 1, max_len, max_len - 1, 7, max_len // 2]
    for Hkv, Hq, B in ((1, 4, 1), (3, 6, 20)):
        s = attn_setup(dt, B, Hq, Hkv, 64, 16, lens, seed=max_len)
        s["pg"] = H.make_page_cfg(16, s["pg"].n_pages, -(-max_len // 16))
        s["table"] = s["table"][:, :s["pg"].max_pages].contiguous()
        check_attn(s, f"up to {max_len} keys")
        one = attn_setup(dt, B, Hq, Hkv, 64, 16, [max_len], seed=1)
        check_attn(one, "one request")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,G", [(1, 1), (3, 1), (1, 4), (1, 5), (7, 1), (2, 4), (1, 8), (9, 1), (3, 3), (1, 11), (5, 3), (4, 4), (1, 16),
                                 (17, 1), (6, 4), (5, 4), (33, 1), (9, 7)])
def test_attention_float32_few_rows(B, G, d):
    """Row counts at which the float32 kernels and the row tiles change; masks of both kinds, requests that are split."""
    for window, sink, scale in ((0, 0, 1.0), (300, 5, 4.0)):
        s = attn_setup(F32, B, 3 * G, 3, d, 16, EDGES + [9000], window, sink, seed=B + 20 * G, k_scale=scale)
        check_attn(s, f"{B} tokens, {G} heads to a key head, window {window}")


@pytest.mark.parametrize("step", [0.0625, 1.0, 32.0])
def test_attention_float32_rising_scores(step):
    """Each key's score is above all before it, by less or by more than what moves the running maximum (8, in log2).

    q = 8, k = j step / 512 in 64 features, both exact: q . k / 8 = j step / 8.  The largest score, in log2, is
    200 * 4 * 1.4427 < 1155, rounded by at most 2^-14 of 1: 6e-5 * ln 2 of a weight, and the weights but the last are below
    2% of it then; with the smaller steps the scores are below 37 and rounded by 2^-19."""
    for B in (1, 2):
        s = attn_setup(F32, B, 4, 1, 64, 128, [200, 129], seed=5)
        for r, x in enumerate(s["lens"].tolist()):
            j = torch.arange(x, device="cuda")
            s["kc"][s["table"][r][j // 128].long(), 0, j % 128] = (j.float() * step / 512.0)[:, None].expand(x, 64)
        s["q"][:] = 8.0
        check_attn(s, f"rising by {step / 8}")
