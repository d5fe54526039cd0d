"""Cases of the operators of an 8-bit paged key-value cache, for the softmax layers of a hybrid model.

A softmax layer in decoding is bound by the bytes of its cache. Three operators hold that cache in 8
bits (e4m3) with a float32 scale, a power of two, for each 16 tokens of a head:

  write   norms of query and key heads with the position rotation, queries to a dense output, keys and
          values rounded into the cache; or keys and values alone, as they are
  read    tokens of the cache, by their slots, as dense keys and values
  attn    attention of one new token, or of an active block of B tokens, over the cache, optionally
          with a window and first tokens that stay visible

Scales: the least power of two (2^-126 at least) that keeps the largest magnitude of the group's
tokens within 448 of it. A call that writes a group's first slot starts the group afresh (tokens of it
that the call does not write become zeros); any other call keeps its tokens, at the larger of the old
scale and the one that the new tokens need.

`run` computes them in their plain form (elementary torch operations) where `own` is false, and through
the framework's entry points where it is true. Lengths are spread evenly over a case's range and put in
an order that the seed chooses, so that a case's work is known without the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
F8 = torch.float8_e4m3fn
EPS = 1e-6
BASE = 10000.0
GROUP = 16          # tokens that share a scale


def listed():
    return [
        # one new token for each request of a batch of 64, behind what its group of 16 holds already
        dict(name="write_token_b64", op="write", dtype="bf16", n=64, new_min=1, new_max=1, start_max=8191, Hq=16, Hkv=4, d=128,
             rot=128, inter=False, norm=True, queries=True, page=16),
        # the active blocks of that batch, 32 tokens each, from wherever the prompt ended
        dict(name="write_block_b64", op="write", dtype="bf16", n=64, new_min=32, new_max=32, start_max=8191, Hq=16, Hkv=4, d=128,
             rot=128, inter=False, norm=True, queries=True, page=32),
        # prompts of every length entering the cache at once
        dict(name="write_prompts_b64", op="write", dtype="bf16", n=64, new_min=1, new_max=2047, start_max=0, Hq=16, Hkv=4, d=128,
             rot=128, inter=False, norm=True, queries=True, page=64),
        # float32 keys and values as they are, from another cache
        dict(name="write_kv_f32", op="write", dtype="f32", n=5, new_min=100, new_max=601, start_max=40, Hq=8, Hkv=8, d=64,
             rot=0, inter=False, norm=False, queries=False, page=16),
        # the last tokens of a few requests, read back in float32
        dict(name="read_tail_f32", op="read", dtype="f32", tok=333, Hkv=4, d=64, page=16),
        # whole contexts read back, as when a request leaves the GPU
        dict(name="read_contexts", op="read", dtype="bf16", tok=150001, Hkv=4, d=128, page=32),
        # one request's next token over a short context: latency
        dict(name="attn_token_b1", op="attn", dtype="bf16", n=1, B=1, Hq=16, Hkv=4, d=128, page=16, len_min=777, len_max=777,
             window=0, sink=0),
        # one new token for each request of a ragged batch
        dict(name="attn_token_b64", op="attn", dtype="bf16", n=64, B=1, Hq=16, Hkv=4, d=128, page=16, len_min=256, len_max=8192,
             window=0, sink=0),
        # the active block of each request of that batch
        dict(name="attn_block_b64", op="attn", dtype="bf16", n=64, B=32, Hq=16, Hkv=4, d=128, page=32, len_min=256,
             len_max=8192, window=0, sink=0),
        # few requests with long contexts, every head with keys of its own
        dict(name="attn_token_long", op="attn", dtype="bf16", n=3, B=1, Hq=16, Hkv=16, d=128, page=64, len_min=100001,
             len_max=131071, window=0, sink=0),
        # small heads, short blocks, a window and first tokens that stay
        dict(name="attn_block_d64", op="attn", dtype="bf16", n=48, B=8, Hq=32, Hkv=8, d=64, page=16, len_min=0, len_max=6001,
             window=4000, sink=20),
        # float32 queries and outputs
        dict(name="attn_token_f32", op="attn", dtype="f32", n=16, B=1, Hq=16, Hkv=4, d=128, page=16, len_min=100, len_max=9000,
             window=0, sink=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["write", "write", "read", "attn", "attn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d, page = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8, 16])
    if op == "read":
        return dict(op=op, dtype=dtype, tok=_log_int(rng, 1, 76_000_000 // (Hkv * d)), Hkv=Hkv, d=d, page=page)
    if op == "write":
        Hq, n = Hkv * rng.choice([1, 2, 4, 5]), _log_int(rng, 1, 128)
        queries = dtype == "bf16" and rng.random() < 0.7
        most = 65000 * 24 * 128 // ((Hq + 2 * Hkv) * d)
        new_max = _log_int(rng, 1, min(4096, max(1, most // n)))
        rot = rng.choice([16, 32, 48, 64] + ([80, 96, 128] if d == 128 else [])) if queries else 0
        return dict(op=op, dtype=dtype, n=n, new_min=rng.randint(1, new_max), new_max=new_max, start_max=_log_int(rng, 1, 16384) - 1,
                    Hq=Hq, Hkv=Hkv, d=d, rot=rot, inter=rng.random() < 0.4, norm=queries and rng.random() < 0.8, queries=queries,
                    page=page)
    G = rng.choice([1, 2, 4, 7, 8])
    B = rng.choice([1, 1, 2, 8, 16, 32, 33, 64])
    n = _log_int(rng, 1, 128)
    # tokens of all contexts together, bounded by the listed cases' bytes and products
    room = 600e6 / (Hkv * d)
    room = min(room, (7e10 if dtype == "bf16" else 1e10) / (4 * d * Hkv * G * B))
    room = min(room, 1.2e9 / (4 * Hkv * G * B))
    len_max = _log_int(rng, 4, max(8, min(131072, int(room / n))))
    windowed = rng.random() < 0.3
    return dict(op=op, dtype=dtype, n=n, B=B, Hq=Hkv * G, Hkv=Hkv, d=d, page=page, len_min=rng.randint(0, len_max), len_max=len_max,
                window=_log_int(rng, 1, max(2, len_max)) if windowed else 0, sink=rng.choice([0, 1, 4, 33, 130]) if windowed else 0)


# ------------------------------------------------------------------ inputs

def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _visible(case, length):
    """Number of visible keys of a context of that length."""
    if case["window"] == 0:
        return length
    lo = max(0, length - case["window"])
    return length - lo + min(case["sink"], lo)


def _exponent(amax):
    """E of the scale 2^E: the least one, -126 at least, with amax <= 448 * 2^E (448 = 0.875 * 2^9)."""
    m, e = torch.frexp(amax)
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126)
    return torch.where(amax > 0, e, torch.full_like(e, -126))


def _power(e):
    """2^e, -126 <= e <= 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _cache(shape, g):
    """Codes and scales of a cache [n_pages, Hkv, page, d] that holds random values, some pages larger than others."""
    n_pages, Hkv, P, d = shape
    codes = torch.empty(shape, dtype=F8, device="cuda")
    scales = torch.empty(n_pages, Hkv, P // GROUP, device="cuda")
    for at in range(0, n_pages, 16384):                    # (bounds the memory of the float32 values)
        part = slice(at, min(at + 16384, n_pages))
        x = torch.randn(codes[part].shape, generator=g, device="cuda")
        x = x * torch.exp2(0.7 * torch.randn(x.shape[0], Hkv, 1, 1, generator=g, device="cuda"))
        x = x.view(-1, Hkv, P // GROUP, GROUP * d)
        s = _power(_exponent(x.abs().amax(-1)))
        codes[part] = (x / s[..., None]).to(F8).view(-1, Hkv, P, d)
        scales[part] = s
    return codes, scales


def prepare(case, seed):
    g, rng = torch.Generator(device="cuda"), random.Random(seed)
    g.manual_seed(seed)
    s = {"case": case}
    {"write": _prepare_write, "read": _prepare_read, "attn": _prepare_attn}[case["op"]](case, s, g, rng)
    if own:
        _prepare_own(case, s)
    return s


def _prepare_write(case, s, g, rng):
    n, Hq, Hkv, d, P, dt = (case[k] for k in ("n", "Hq", "Hkv", "d", "page", "dtype"))
    order, dt = list(range(n)), DT[dt]
    rng.shuffle(order)
    new = [_spread(case["new_min"], case["new_max"], n)[i] for i in order]
    start = [rng.randint(0, case["start_max"]) for _ in range(n)]
    # the pages that the new tokens are written to, in any order; the others of a request are not in this pool
    first, pages = [x // P for x in start], [(x + k - 1) // P - x // P + 1 for x, k in zip(start, new)]
    T, s["n_pages"] = sum(new), sum((k + 2 * P - 2) // P for k in new) + 3     # enough wherever they start
    ids = np.random.RandomState(rng.getrandbits(31)).permutation(s["n_pages"])
    of = np.repeat(np.arange(n), new)
    pos = np.concatenate([np.arange(x, x + k) for x, k in zip(start, new)])
    slots = ids[(np.cumsum(pages) - pages)[of] + pos // P - np.array(first)[of]] * P + pos % P
    i32 = lambda v: torch.from_numpy(np.ascontiguousarray(v, dtype=np.int32)).cuda()  # noqa: E731
    s["pos"], s["slots"] = i32(pos), i32(slots)
    width = (Hq if case["queries"] else 0) + 2 * Hkv
    qkv = torch.randn(T, width * d, generator=g, device="cuda").to(dt).view(T, width, d)      # one projection's output
    s["q"] = qkv[:, :width - 2 * Hkv] if case["queries"] else None
    s["k"], s["v"] = qkv[:, width - 2 * Hkv:width - Hkv], qkv[:, width - Hkv:]
    w = (1 + 0.1 * torch.randn(2, d, generator=g, device="cuda")).to(dt)
    s["wq"], s["wk"] = (w[0], w[1]) if case["norm"] else (None, None)
    for x in ("k", "v"):
        s[x + "_cache"], s[x + "_scale"] = _cache((s["n_pages"], Hkv, P, d), g)


def _prepare_read(case, s, g, rng):
    T, Hkv, d, P = (case[k] for k in ("tok", "Hkv", "d", "page"))
    s["n_pages"] = -(-T // P) + 5
    page = torch.randperm(s["n_pages"], generator=g, device="cuda")[:-(-T // P)]
    t = torch.arange(T, device="cuda")
    s["slots"] = (page[t // P] * P + t % P).to(torch.int32)
    for x in ("k", "v"):
        s[x + "_cache"], s[x + "_scale"] = _cache((s["n_pages"], Hkv, P, d), g)


def _prepare_attn(case, s, g, rng):
    n, B, Hq, Hkv, d, P = (case[k] for k in ("n", "B", "Hq", "Hkv", "d", "page"))
    order = list(range(n))
    rng.shuffle(order)
    lens = [_spread(case["len_min"], case["len_max"], n)[i] for i in order]
    max_pages = max(1, -(-max(lens) // P))
    used = np.array([-(-x // P) for x in lens])
    s["n_pages"], s["max_pages"] = int(used.sum()) + 3, max_pages
    ids = np.random.RandomState(rng.getrandbits(31)).permutation(s["n_pages"])
    table = np.full((n, max_pages), -1, dtype=np.int32)
    table[np.arange(max_pages)[None, :] < used[:, None]] = ids[:used.sum()]
    s["table"], s["lens"] = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    s["q"] = torch.randn(n, B, Hq, d, generator=g, device="cuda").to(DT[case["dtype"]])
    for x in ("k", "v"):
        s[x + "_cache"], s[x + "_scale"] = _cache((s["n_pages"], Hkv, P, d), g)


def _prepare_own(case, s):
    """What a user of the framework keeps: configurations, output buffers and workspaces."""
    from paper_2608_06628_gb300 import hybrid as H
    s["H"], dt, d, Hkv = H, DT[case["dtype"]], case["d"], case["Hkv"]
    s["cfg"] = H.make_cfg(d, 64, case.get("Hq", Hkv), Hkv, case.get("B", 1), dt)
    s["pg"] = H.make_page_cfg(case["page"], s["n_pages"], s.get("max_pages", 1))
    if case["op"] == "write":
        s["rope"], s["freqs"] = H.make_rope(case["rot"], case["inter"], eps=EPS, base=BASE, device="cuda")
        s["qo"] = torch.empty(s["q"].shape, dtype=dt, device="cuda") if case["queries"] else None
    elif case["op"] == "read":
        s["k"], s["v"] = torch.empty(2, case["tok"], Hkv, d, dtype=dt, device="cuda")
    else:
        s["o"] = torch.empty_like(s["q"])
        s["ws_bytes"] = H.hybrid_paged_attn_quant_workspace_bytes(s["cfg"], s["pg"], case["n"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass

def run(state):
    return {"write": _write, "read": _read, "attn": _attn}[state["case"]["op"]](state)


def _norm_rotate(x, w, s):
    """In 64 bits: keys stand next to the borders of 8-bit values, and angles of far positions lose theirs in 32."""
    c, x = s["case"], x.double()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.double()
    rot = c["rot"]
    if rot == 0:
        return x
    turn = torch.exp(torch.arange(0, rot, 2, device=x.device, dtype=torch.float64) * (-math.log(BASE) / rot))
    ang = s["pos"].double()[:, None, None] * turn
    cos, sin, rest = torch.cos(ang), torch.sin(ang), x[..., rot:]
    if c["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
    a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _put(cache, scale, x, slots):
    """x [T, Hkv, d] (64 bits) into the cache's slots: the cache and its scales, in place."""
    n_pages, Hkv, P, d = cache.shape
    T, per = x.shape[0], P // GROUP
    slots = slots.long()
    group, off = slots // GROUP, slots % GROUP
    n = n_pages * per
    amax = torch.zeros(n, Hkv, dtype=x.dtype, device=x.device)
    amax.scatter_reduce_(0, group[:, None].expand(T, Hkv), x.abs().amax(-1), "amax")
    need = _exponent(amax)
    written = torch.zeros(n, GROUP, dtype=torch.bool, device=x.device)
    written[group, off] = True
    touched, fresh = written.any(1)[:, None], written[:, :1]
    old = scale.permute(0, 2, 1).reshape(n, Hkv)
    has = torch.frexp(old)[1] - 1
    e = torch.where(fresh, need, torch.maximum(need, has))
    e = torch.where(touched, e, has)
    # tokens that the call does not write: their value at the new scale, or zero
    codes = cache.view(n_pages, Hkv, per, GROUP, d).permute(0, 2, 3, 1, 4).reshape(n, GROUP, Hkv, d).float()
    keep = codes * _power((has - e).clamp(min=-126))[:, None, :, None]
    keep = torch.where((touched & fresh)[:, None, :, None], torch.zeros((), device=x.device), keep)
    keep[group, off] = (x * _power(-e)[group][..., None].double()).float()
    cache.copy_(keep.to(F8).view(n_pages, per, GROUP, Hkv, d).permute(0, 3, 1, 2, 4).reshape(cache.shape))
    scale.copy_(_power(e).view(n_pages, per, Hkv).permute(0, 2, 1))


def _write(s):
    c = s["case"]
    if own:
        H, q = s["H"], s["q"]
        H.hybrid_qk_norm_rope_cache_quant(s["cfg"], s["rope"], s["pg"], q, q.stride(0) if q is not None else 0, s["k"],
                                          s["k"].stride(0), s["v"], s["v"].stride(0), s["k"].shape[0], s["wq"], s["wk"], s["pos"],
                                          s["freqs"], s["slots"], s["qo"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        out = {"q": s["qo"]} if c["queries"] else {}
    else:
        out = {"q": _norm_rotate(s["q"], s["wq"], s).to(DT[c["dtype"]])} if c["queries"] else {}
        _put(s["k_cache"], s["k_scale"], _norm_rotate(s["k"], s["wk"], s), s["slots"])
        _put(s["v_cache"], s["v_scale"], s["v"].double(), s["slots"])
    out.update(k_cache=s["k_cache"], v_cache=s["v_cache"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    return out


def _read(s):
    c = s["case"]
    if own:
        s["H"].hybrid_cache_dequant(s["cfg"], s["pg"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["slots"], c["tok"],
                                    s["k"], s["v"])
        return {"k": s["k"], "v": s["v"]}
    page, off, out = s["slots"].long() // c["page"], s["slots"].long() % c["page"], {}
    for x in ("k", "v"):
        codes = s[x + "_cache"].view(torch.uint8)[page, :, off].view(F8).float()
        out[x] = (codes * s[x + "_scale"][page, :, off // GROUP][..., None]).to(DT[c["dtype"]])
    return out


def _attn(s):
    c = s["case"]
    if own:
        s["H"].hybrid_paged_attn_quant(s["cfg"], s["pg"], s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"],
                                       s["lens"], c["n"], c["window"], c["sink"], s["o"], s["ws"], s["ws_bytes"])
        return s["o"]
    n, B, Hq, Hkv, d, P = (c[k] for k in ("n", "B", "Hq", "Hkv", "d", "page"))
    L = s["max_pages"] * P
    pages = s["table"].long().clamp(min=0)

    def gather(x):
        codes = s[x + "_cache"].view(torch.uint8)[pages].transpose(1, 2).reshape(n, Hkv, -1, GROUP, d).view(F8).float()
        return (codes * s[x + "_scale"][pages].transpose(1, 2).reshape(n, Hkv, -1, 1, 1)).reshape(n, Hkv, L, d)

    at, lens = torch.arange(L, device=s["lens"].device), s["lens"].long()[:, None]
    see = at < lens
    if c["window"]:
        see = see & ((at >= lens - c["window"]) | (at < c["sink"]))
    q = s["q"].float().view(n, B, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d)
    x = q @ gather("k").transpose(-1, -2) * (1.0 / math.sqrt(d))
    x = torch.where(see[:, None, None, :], x, torch.full((), -math.inf, device=x.device))
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    v = torch.where(see[:, None, :, None], gather("v"), torch.zeros((), device=x.device))
    o = (x @ v) / x.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(n, Hkv, B, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, B, Hq, d).to(DT[c["dtype"]])


# ------------------------------------------------------------------ work and exact values

def work(case):
    d, Hkv, es = case["d"], case["Hkv"], ES[case["dtype"]]
    if case["op"] == "attn":
        seen = sum(_visible(case, x) for x in _spread(case["len_min"], case["len_max"], case["n"]))
        rows = case["n"] * case["B"] * case["Hq"]
        return {"bytes": seen * Hkv * (2 * d + 8 / GROUP) + es * 2 * rows * d + 4 * (seen // case["page"] + case["n"]),
                "flops": 4 * seen * case["Hq"] * case["B"] * d}
    if case["op"] == "read":
        return {"bytes": case["tok"] * (Hkv * ((1 + es) * 2 * d + 8 / GROUP) + 4), "flops": 2 * case["tok"] * Hkv * d}
    T = sum(_spread(case["new_min"], case["new_max"], case["n"]))
    Hq = case["Hq"] if case["queries"] else 0
    return {"bytes": T * ((es * (2 * Hq + 2 * Hkv) + 2 * Hkv) * d + 8 * Hkv / GROUP + (8 if case["rot"] else 4)),
            "flops": T * (8 * (Hq + Hkv) + 2 * Hkv) * d if case["rot"] or case["norm"] else 4 * T * Hkv * d}


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"write": _exact_write, "read": _exact_read, "attn": _exact_attn}[case["op"]](case, s)


def _exact_write(case, s):
    """Codes before their rounding, token by token of the touched groups; the queries as complex rotations."""
    rot, P, d, Hkv = case["rot"], case["page"], case["d"], case["Hkv"]
    if s["slots"].numel() * Hkv * d > 4_000_000:
        return None

    def formed(x, w):
        x = x.double()
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + EPS) * w.double()
        if rot:
            i = torch.arange(rot // 2, device=x.device, dtype=torch.float64)
            z = torch.polar(torch.ones((), device=x.device, dtype=torch.float64),
                            s["pos"].double()[:, None, None] * torch.pow(torch.full_like(i, BASE), -2 * i / rot))
            a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["inter"] else (x[..., :rot // 2], x[..., rot // 2:rot])
            y, x = torch.complex(a, b) * z, x.clone()
            if case["inter"]:
                x[..., 0:rot:2], x[..., 1:rot:2] = y.real, y.imag
            else:
                x[..., :rot // 2], x[..., rot // 2:rot] = y.real, y.imag
        return x.cpu().numpy()

    slots = s["slots"].cpu().numpy()
    members = {}
    for t, slot in enumerate(slots.tolist()):
        members.setdefault(slot // GROUP, []).append(t)
    out = {"q": formed(s["q"], s["wq"])} if case["queries"] else {}
    for name, x in (("k", formed(s["k"], s["wk"])), ("v", s["v"].double().cpu().numpy())):
        cache, scale = s[name + "_cache"].double().cpu().numpy(), s[name + "_scale"].double().cpu().numpy()
        for group, ts in members.items():
            page, at = divmod(group * GROUP, P)
            offs = slots[ts] % GROUP
            new = x[ts]                                       # [tokens, Hkv, d]
            top = np.abs(new).max(axis=(0, 2))
            need = np.exp2(np.maximum(np.ceil(np.log2(np.where(top > 0, top, 1.0) / 448.0)), -126))
            need = np.where(top > 0, need, 2.0 ** -126)
            held = cache[page, :, at:at + GROUP]              # [Hkv, tokens, d], a view
            if 0 in offs:
                held[:] = 0.0
            else:
                need = np.maximum(need, scale[page, :, at // GROUP])
                held *= (scale[page, :, at // GROUP] / need)[:, None, None]
            held[:, offs] = new.transpose(1, 0, 2) / need[:, None, None]
            scale[page, :, at // GROUP] = need
        out[name + "_cache"], out[name + "_scale"] = cache, scale
    keys = (["q"] if case["queries"] else []) + ["k_cache", "v_cache", "k_scale", "v_scale"]
    return {k: out[k] for k in keys}


def _exact_read(case, s):
    P, slots, out = case["page"], s["slots"].cpu().numpy(), {}
    if slots.size * case["Hkv"] * case["d"] > 4_000_000:
        return None
    for x in ("k", "v"):
        codes, scale = s[x + "_cache"].double().cpu().numpy(), s[x + "_scale"].double().cpu().numpy()
        out[x] = np.stack([codes[t // P, :, t % P] * scale[t // P, :, t % P // GROUP, None] for t in slots.tolist()])
    return out


def _exact_attn(case, s):
    n, B, Hq, Hkv, d, P = (case[k] for k in ("n", "B", "Hq", "Hkv", "d", "page"))
    seen = sum(_visible(case, x) for x in _spread(case["len_min"], case["len_max"], n))
    if 4.0 * seen * Hq * B * d > 1.5e12:
        return None
    G, out = Hq // Hkv, torch.zeros(n, B, Hq, d, dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["lens"].tolist()):
        keys = list(range(length))
        if case["window"]:
            lo = max(0, length - case["window"])
            keys = list(range(min(case["sink"], lo))) + list(range(lo, length))
        if not keys:
            continue
        j = torch.tensor(keys, device="cuda")
        page, at = s["table"][r, j // P].long(), j % P
        for h in range(Hkv):
            k, v = (s[x + "_cache"].view(torch.uint8)[page, h, at].view(F8).double() *
                    s[x + "_scale"][page, h, at // GROUP].double()[:, None] for x in ("k", "v"))
            for g in range(h * G, h * G + G):
                out[r, :, g] = torch.softmax(s["q"][r, :, g].double() @ k.T / math.sqrt(d), -1) @ v
    return out.cpu().numpy()
