"""Cases of the operators that the softmax layers of a hybrid model run beside the block-hybrid ones.

A retrofitted model keeps most of its layers on exact attention over a paged key-value cache. Four
operators carry such a layer through a denoising step:

  pages      block tables and slot maps built on the device from request lengths (pages taken from a
             ring of free pages for the new tokens, and given back for finished requests)
  rope       norms of the queries and keys of each head with the position rotation, in one pass,
             into dense outputs or straight into the paged cache
  rope_bwd   the gradient of that pass: inputs and norm weights
  attn       attention of one new token, or of an active block of B tokens, over the paged cache,
             optionally with a window and first tokens that stay visible

`run` computes them in their plain form (elementary torch operations in 32 bits) where `own` is
false, and through the framework's entry points where it is true. A case's lengths are spread evenly
over its range and put in an order that the seed chooses, so that its work is known without the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # the start of a block for a serving batch: 32 new tokens for each of 64 requests, 4 of them finished
        dict(name="pages_block_b64", op="pages", n=64, page=16, len_min=256, len_max=8192, new_min=32, new_max=32, done=4),
        # prompts of every length entering a large pool at once
        dict(name="pages_prompts_b1000", op="pages", n=1000, page=64, len_min=0, len_max=1000, new_min=1, new_max=2047, done=300),
        # one new token per request of a batch of 64, written to the cache
        dict(name="rope_token_b64", op="rope", dtype="bf16", tok=64, Hq=16, Hkv=4, d=128, rot=128, inter=False, norm=True,
             cache=True, page=16, scaling="none", max_pos=8192),
        # the active blocks of that batch: 64 x 32 tokens, written to the cache
        dict(name="rope_block_b64", op="rope", dtype="bf16", tok=2048, Hq=16, Hkv=4, d=128, rot=128, inter=False, norm=True,
             cache=True, page=32, scaling="yarn", max_pos=131072),
        # long prompts, float32, interleaved pairs on half of each head
        dict(name="rope_prompt_f32", op="rope", dtype="f32", tok=20011, Hq=16, Hkv=16, d=64, rot=32, inter=True, norm=True,
             cache=False, page=16, scaling="linear", max_pos=32768),
        # a training batch of 8 sequences of 2048 tokens
        dict(name="rope_bwd_8x2048", op="rope_bwd", dtype="bf16", tok=16384, Hq=16, Hkv=4, d=128, rot=128, inter=False,
             norm=True, scaling="none", max_pos=2048),
        # a short float32 training sequence
        dict(name="rope_bwd_f32_short", op="rope_bwd", dtype="f32", tok=321, Hq=2, Hkv=2, d=64, rot=48, inter=True,
             norm=True, scaling="ntk", max_pos=8192),
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
        # float32, an active block of 16 with a window and first tokens that stay
        dict(name="attn_window_f32", op="attn", dtype="f32", n=8, B=16, Hq=8, Hkv=2, d=64, page=16, len_min=100, len_max=9000,
             window=2000, sink=20),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "rope", "rope_bwd", "attn", "attn"])
    if op == "pages":
        n = _log_int(rng, 1, 2000)
        new_max = _log_int(rng, 1, min(2048, 1000000 // n))
        len_max = _log_int(rng, 1, 16384)
        return dict(op=op, n=n, page=rng.choice([16, 32, 64, 128]), len_min=rng.randint(0, len_max), len_max=len_max,
                    new_min=rng.randint(0, new_max), new_max=new_max, done=rng.randint(0, n))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8, 16])
    if op != "attn":
        Hq = Hkv * rng.choice([1, 2, 4, 5])
        c = dict(op=op, dtype=dtype, tok=_log_int(rng, 1, max(2, 16384 * 20 // (Hq + Hkv))), Hq=Hq, Hkv=Hkv, d=d,
                 rot=rng.choice([16, 32, 48, 64] + ([80, 96, 128] if d == 128 else [])), inter=rng.random() < 0.5,
                 norm=rng.random() < 0.8, scaling=rng.choice(["none", "linear", "ntk", "yarn"]),
                 max_pos=_log_int(rng, 128, 131072))
        if op == "rope":
            c.update(cache=rng.random() < 0.6, page=rng.choice([16, 32, 64, 128]))
        return c
    G = rng.choice([1, 2, 4, 7, 8])
    B = rng.choice([1, 1, 2, 16, 32, 33, 64])
    n = _log_int(rng, 1, 128)
    # tokens of all contexts together, bounded by the listed cases' bytes and products
    room = 800e6 / (Hkv * d * 2 * ES[dtype])
    room = min(room, (7e10 if dtype == "bf16" else 2e10) / (4 * d * Hkv * G * B))
    room = min(room, 1.2e9 / (4 * Hkv * G * B))
    len_max = _log_int(rng, 4, max(8, min(131072, int(room / n))))
    windowed = rng.random() < 0.3
    return dict(op=op, dtype=dtype, n=n, B=B, Hq=Hkv * G, Hkv=Hkv, d=d, page=rng.choice([16, 32, 64, 128]),
                len_min=rng.randint(0, len_max), len_max=len_max, window=_log_int(rng, 1, max(2, len_max)) if windowed else 0,
                sink=rng.choice([0, 1, 4, 33, 130]) if windowed else 0)


# ------------------------------------------------------------------ inputs

def _spread(lo, hi, n):
    """n whole numbers spread evenly over [lo, hi]."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lens(case, order):
    return [_spread(case["len_min"], case["len_max"], case["n"])[i] for i in order]


def _visible(case, length):
    """Number of visible keys of a context of that length."""
    if case["window"] == 0:
        return length
    lo = max(0, length - case["window"])
    return length - lo + min(case["sink"], lo)


def _turns(case):
    """Turns per position of each pair of features, and the factor on cosine and sine."""
    rot, kind, factor, orig = case["rot"], case["scaling"], 4.0, 4096.0
    base = BASE * factor ** (rot / (rot - 2)) if kind == "ntk" else BASE
    out = []
    for i in range(rot // 2):
        t = base ** (-2.0 * i / rot) / (2.0 * math.pi)
        if kind == "linear":
            t /= factor
        elif kind == "yarn":
            keep = min(1.0, max(0.0, (orig * t - 1.0) / (32.0 - 1.0)))
            t = t / factor * (1.0 - keep) + t * keep
        out.append(t)
    return out, (0.1 * math.log(factor) + 1.0 if kind == "yarn" else 1.0)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g, rng = _gen(seed), random.Random(seed)
    s = {"case": case}
    if case["op"] == "pages":
        _prepare_pages(case, s, rng)
    elif case["op"] == "attn":
        _prepare_attn(case, s, g, rng)
    else:
        _prepare_rope(case, s, g)
    if own:
        _prepare_own(case, s)
    return s


def _prepare_pages(case, s, rng):
    n, P = case["n"], case["page"]
    order, order2 = list(range(n)), list(range(n))
    rng.shuffle(order)
    rng.shuffle(order2)
    lens = _lens(case, order)
    new = [_spread(case["new_min"], case["new_max"], n)[i] for i in order2]
    max_pages = -(-(case["len_max"] + case["new_max"]) // P)
    held = sum(-(-x // P) for x in lens)
    n_pages = held + sum(new) // P + n + 7                 # enough for any pairing of lengths and new tokens
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(rng.getrandbits(40))).to(torch.int32)
    table = torch.full((n, max_pages), -1, dtype=torch.int32)
    at = 0
    for r, x in enumerate(lens):
        k = -(-x // P)
        table[r, :k] = ids[at:at + k]
        at += k
    head, count = rng.randrange(n_pages), n_pages - held
    free = torch.full((n_pages,), -1, dtype=torch.int32)
    free[(head + torch.arange(count)) % n_pages] = ids[held:]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    total = sum(new)
    s.update(n_pages=n_pages, max_pages=max_pages, n_slots=-(-max(total, 1) // 256) * 256, lens=i32(lens), new=i32(new),
             table=table.cuda(), free=free.cuda(), ring=i32([head, count]), rows=i32(rng.sample(range(n), case["done"])))


def _prepare_rope(case, s, g):
    T, Hq, Hkv, d, rot, dt = case["tok"], case["Hq"], case["Hkv"], case["d"], case["rot"], DT[case["dtype"]]
    qkv = torch.randn(T, (Hq + 2 * Hkv) * d, generator=g, device="cuda").to(dt)   # one projection's output
    s["q"] = qkv[:, :Hq * d].view(T, Hq, d)
    s["k"] = qkv[:, Hq * d:(Hq + Hkv) * d].view(T, Hkv, d)
    s["v"] = qkv[:, (Hq + Hkv) * d:].view(T, Hkv, d)
    w = (1 + 0.1 * torch.randn(2, d, generator=g, device="cuda")).to(dt)
    s["wq"], s["wk"] = (w[0], w[1]) if case["norm"] else (None, None)
    s["pos"] = torch.randint(0, case["max_pos"], (T,), generator=g, device="cuda", dtype=torch.int32)
    if case["op"] == "rope_bwd":
        s["dy"] = torch.randn(T, Hq * d, generator=g, device="cuda").to(dt).view(T, Hq, d)
        s["dk"] = torch.randn(T, Hkv * d, generator=g, device="cuda").to(dt).view(T, Hkv, d)
    if case.get("cache"):
        P = case["page"]
        s["n_pages"] = -(-T // P) + 5
        slots = torch.randperm(s["n_pages"] * P, generator=g, device="cuda")[:T].to(torch.int32)
        slots[torch.rand(T, generator=g, device="cuda") < 0.03] = -1       # padding of a fixed-size batch
        s["slots"] = slots
        kv = torch.randn(2, s["n_pages"], Hkv, P, d, generator=g, device="cuda").to(dt)
        s["k_cache"], s["v_cache"] = kv[0], kv[1]
    if not own:
        turns, scale = _turns(case)
        ang = torch.arange(case["max_pos"], device="cuda", dtype=torch.float64)[:, None] * \
            torch.tensor(turns, device="cuda", dtype=torch.float64)[None, :] * (2 * math.pi)
        s["cos"], s["sin"] = (torch.cos(ang) * scale).float(), (torch.sin(ang) * scale).float()


def _prepare_attn(case, s, g, rng):
    n, B, Hq, Hkv, d, P, dt = (case[k] for k in ("n", "B", "Hq", "Hkv", "d", "page", "dtype"))
    order = list(range(n))
    rng.shuffle(order)
    lens = _lens(case, order)
    max_pages = max(1, -(-max(lens) // P))
    used = [-(-x // P) for x in lens]
    n_pages = sum(used) + 3
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(rng.getrandbits(40))).to(torch.int32)
    table = torch.full((n, max_pages), -1, dtype=torch.int32)
    at = 0
    for r, k in enumerate(used):
        table[r, :k] = ids[at:at + k]
        at += k
    s.update(n_pages=n_pages, max_pages=max_pages, table=table.cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    s["q"] = torch.randn(n, B, Hq, d, generator=g, device="cuda").to(DT[dt])
    s["k_cache"] = torch.randn(n_pages, Hkv, P, d, generator=g, device="cuda", dtype=DT[dt])
    s["v_cache"] = torch.randn(n_pages, Hkv, P, d, generator=g, device="cuda", dtype=DT[dt])


def _prepare_own(case, s):
    """What a user of the framework keeps: configurations, output buffers and workspaces."""
    from paper_2608_06628_gb300 import hybrid as H
    s["H"] = H
    if case["op"] == "pages":
        i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")  # noqa: E731
        s["pg"] = H.make_page_cfg(case["page"], s["n_pages"], s["max_pages"])
        s.update(slots=i32(s["n_slots"]), pos=i32(s["n_slots"]), offs=i32(case["n"] + 1), lens_out=i32(case["n"]),
                 ring_mid=i32(2), ring_out=i32(2))
        return
    cfg = H.make_cfg(case["d"], 64, case["Hq"], case["Hkv"], case.get("B", 1), DT[case["dtype"]])
    s["cfg"] = cfg
    if case["op"] == "attn":
        s["pg"] = H.make_page_cfg(case["page"], s["n_pages"], s["max_pages"])
        s["o"] = torch.empty_like(s["q"])
        s["ws_bytes"] = H.hybrid_paged_attn_workspace_bytes(cfg, s["pg"], case["n"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")
        return
    kind = {"none": H.HYBRID_ROPE_NONE, "linear": H.HYBRID_ROPE_LINEAR, "ntk": H.HYBRID_ROPE_NTK, "yarn": H.HYBRID_ROPE_YARN}
    s["rope"], s["freqs"] = H.make_rope(case["rot"], case["inter"], eps=EPS, base=BASE, kind=kind[case["scaling"]],
                                        factor=4.0, orig_len=4096.0, device="cuda")
    T, Hq, Hkv, d, dt = case["tok"], case["Hq"], case["Hkv"], case["d"], DT[case["dtype"]]
    if case["op"] == "rope":
        s["qo"] = torch.empty(T, Hq, d, dtype=dt, device="cuda")
        if case["cache"]:
            s["pg"] = H.make_page_cfg(case["page"], s["n_pages"], 1)
        else:
            s["ko"] = torch.empty(T, Hkv, d, dtype=dt, device="cuda")
    else:
        dqkv = torch.empty(T, (Hq + 2 * Hkv) * d, dtype=dt, device="cuda")     # the projection's gradient
        s["gq"], s["gk"] = dqkv[:, :Hq * d].view(T, Hq, d), dqkv[:, Hq * d:(Hq + Hkv) * d].view(T, Hkv, d)
        s["gwq"], s["gwk"] = (torch.empty(2, d, dtype=torch.float32, device="cuda")) if case["norm"] else (None, None)
        s["ws_bytes"] = H.hybrid_qk_norm_rope_workspace_bytes(cfg, T)
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ one pass

def run(state):
    return {"pages": _pages, "rope": _rope, "rope_bwd": _rope_bwd, "attn": _attn}[state["case"]["op"]](state)


def _pages(s):
    c, n = s["case"], s["case"]["n"]
    if own:
        H = s["H"]
        H.hybrid_page_append(s["pg"], n, s["lens"], s["new"], s["free"], s["ring"], s["table"], s["slots"], s["pos"],
                             s["n_slots"], s["offs"], s["lens_out"], s["ring_mid"])
        H.hybrid_page_release(s["pg"], n, s["rows"], c["done"], s["lens_out"], s["table"], s["free"], s["ring_mid"],
                              s["ring_out"])
        return {"table": s["table"], "slots": s["slots"], "pos": s["pos"], "offs": s["offs"], "lens": s["lens_out"],
                "free": s["free"], "ring": s["ring_out"]}
    P, N, dev = c["page"], s["n_pages"], s["lens"].device
    lens, new, table, free = s["lens"].long(), s["new"].long(), s["table"], s["free"]
    old = (lens + P - 1) // P
    need = (lens + new + P - 1) // P - old
    first = torch.cumsum(need, 0) - need
    offs = torch.zeros(n + 1, dtype=torch.int64, device=dev)
    offs[1:] = torch.cumsum(new, 0)
    t = torch.arange(s["n_slots"], device=dev)
    real = t < offs[n]
    t = torch.where(real, t, torch.zeros_like(t))          # padding repeats the first token's work
    r = (torch.searchsorted(offs, t, right=True) - 1).clamp(max=n - 1)
    p = lens[r] + t - offs[r]
    j = (p // P).clamp(max=table.shape[1] - 1)
    fresh = (offs[n] > 0) & (j >= old[r])
    taken = free[(s["ring"][0] + first[r] + j - old[r]) % N]
    page = torch.where(fresh, taken, table[r, j])
    slots = torch.where(real, page * P + p % P, torch.full_like(t, -1))
    table[r, j] = page                                     # every token of a page writes the same entry
    lens_out = lens + new
    used = need.sum()
    head, count = (s["ring"][0] + used) % N, s["ring"][1] - used
    rows = s["rows"].long()
    k = (lens_out[rows] + P - 1) // P
    at = torch.cumsum(k, 0) - k
    col = torch.arange(table.shape[1], device=dev)
    give = col[None, :] < k[:, None]
    where = (head + count + at[:, None] + col[None, :]) % N
    scratch = torch.cat([free, free[:1]])
    scratch[torch.where(give, where, torch.full_like(where, N))] = table[rows]
    free.copy_(scratch[:N])
    ring = torch.stack([head, count + k.sum()])
    return {"table": table, "slots": slots.int(), "pos": torch.where(real, p, torch.zeros_like(p)).int(), "offs": offs.int(), "lens": lens_out.int(), "free": free,
            "ring": ring.int()}


def _split(x, case):
    """The two members of each rotated pair, and what is not rotated."""
    rot = case["rot"]
    if case["inter"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _join(a, b, rest, case):
    if case["inter"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _norm_rotate(x, w, s):
    x = x.float()
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    a, b, rest = _split(x, s["case"])
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    return _join(a * cos - b * sin, b * cos + a * sin, rest, s["case"])


def _rope(s):
    c = s["case"]
    if own:
        H, T = s["H"], c["tok"]
        if c["cache"]:
            H.hybrid_qk_norm_rope_cache(s["cfg"], s["rope"], s["pg"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0),
                                        s["v"], s["v"].stride(0), T, s["wq"], s["wk"], s["pos"], s["freqs"], s["slots"],
                                        s["qo"], s["k_cache"], s["v_cache"])
            return {"q": s["qo"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        H.hybrid_qk_norm_rope(s["cfg"], s["rope"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), T, s["wq"], s["wk"],
                              s["pos"], s["freqs"], s["qo"], s["ko"])
        return {"q": s["qo"], "k": s["ko"]}
    dt = DT[c["dtype"]]
    q, k = _norm_rotate(s["q"], s["wq"], s).to(dt), _norm_rotate(s["k"], s["wk"], s).to(dt)
    if not c["cache"]:
        return {"q": q, "k": k}
    P, spare = c["page"], s["n_pages"]
    slot = s["slots"].long()
    page = torch.where(slot < 0, torch.full_like(slot, spare), slot // P)      # padding goes to a page that is dropped
    out = {"q": q}
    for name, x in (("k_cache", k), ("v_cache", s["v"])):
        cache = torch.cat([s[name], torch.zeros_like(s[name][:1])])
        cache[page, :, slot % P] = x
        s[name].copy_(cache[:spare])
        out[name] = s[name]
    return out


def _grad(x, w, dy, s):
    """Gradients of sum(dy * norm_rotate(x, w)) in x and w."""
    x, (a, b, rest) = x.float(), _split(dy.float(), s["case"])
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    dn = _join(a * cos + b * sin, b * cos - a * sin, rest, s["case"])
    if w is None:
        return dn, None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xh, u = x * r, dn * w.float()
    return r * (u - xh * (u * xh).mean(-1, keepdim=True)), (dn * xh).sum((0, 1))


def _rope_bwd(s):
    c = s["case"]
    if own:
        s["H"].hybrid_qk_norm_rope_backward(s["cfg"], s["rope"], s["q"], s["q"].stride(0), s["k"], s["k"].stride(0), s["dy"],
                                            s["dk"], c["tok"], s["wq"], s["wk"], s["pos"], s["freqs"], s["ws"], s["ws_bytes"],
                                            s["gq"], s["gk"], s["gwq"], s["gwk"])
        out = {"dq": s["gq"], "dk": s["gk"]}
        if c["norm"]:
            out.update(dwq=s["gwq"], dwk=s["gwk"])
        return out
    dt = DT[c["dtype"]]
    (dq, dwq), (dk, dwk) = _grad(s["q"], s["wq"], s["dy"], s), _grad(s["k"], s["wk"], s["dk"], s)
    out = {"dq": dq.to(dt), "dk": dk.to(dt)}
    if c["norm"]:
        out.update(dwq=dwq, dwk=dwk)
    return out


def _attn(s):
    c = s["case"]
    if own:
        s["H"].hybrid_paged_attn(s["cfg"], s["pg"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], c["n"],
                                 c["window"], c["sink"], s["o"], s["ws"], s["ws_bytes"])
        return s["o"]
    n, B, Hq, Hkv, d, P = (c[k] for k in ("n", "B", "Hq", "Hkv", "d", "page"))
    L = s["max_pages"] * P
    pages = s["table"].long().clamp(min=0)
    gather = lambda x: x[pages].transpose(1, 2).reshape(n, Hkv, L, d).float()  # noqa: E731
    at = torch.arange(L, device=s["lens"].device)
    lens = s["lens"].long()[:, None]
    see = at < lens
    if c["window"]:
        see = see & ((at >= lens - c["window"]) | (at < c["sink"]))
    q = s["q"].float().view(n, B, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d)
    x = q @ gather(s["k_cache"]).transpose(-1, -2) * (1.0 / math.sqrt(d))
    x = torch.where(see[:, None, None, :], x, torch.full((), -math.inf, device=x.device))
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    v = torch.where(see[:, None, :, None], gather(s["v_cache"]), torch.zeros((), device=x.device))
    o = (x @ v) / x.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(n, Hkv, B, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, B, Hq, d).to(DT[c["dtype"]])


# ------------------------------------------------------------------ work and exact values

def work(case):
    if case["op"] == "pages":
        n, P = case["n"], case["page"]
        total = sum(_spread(case["new_min"], case["new_max"], n))
        slots = -(-max(total, 1) // 256) * 256
        moved = total // P + case["done"] * ((case["len_min"] + case["len_max"] + case["new_min"] + case["new_max"]) // (2 * P))
        return {"bytes": 4 * (4 * n + 2 * slots + 2 * moved), "flops": 0}
    d, Hq, Hkv, es = case["d"], case["Hq"], case["Hkv"], ES[case["dtype"]]
    if case["op"] == "attn":
        seen = sum(_visible(case, x) for x in _spread(case["len_min"], case["len_max"], case["n"]))
        rows = case["n"] * case["B"] * Hq
        return {"bytes": es * (2 * seen * Hkv * d + 2 * rows * d) + 4 * (seen // case["page"] + case["n"]),
                "flops": 4 * seen * Hq * case["B"] * d}
    rows = case["tok"] * (Hq + Hkv)
    if case["op"] == "rope":
        moved = 2 * rows + (2 * case["tok"] * Hkv if case["cache"] else 0)
        return {"bytes": es * moved * d + 8 * case["tok"], "flops": 8 * rows * d}
    return {"bytes": es * (3 if case["norm"] else 2) * rows * d + 4 * case["tok"], "flops": 16 * rows * d}


def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    return {"pages": _exact_pages, "rope": _exact_rope, "rope_bwd": _exact_rope, "attn": _exact_attn}[case["op"]](case, s)


def _exact_pages(case, s):
    """The pool's rules, one token at a time."""
    P, N = case["page"], s["n_pages"]
    table, free = s["table"].cpu().numpy().copy(), s["free"].cpu().numpy().copy()
    head, count = (int(x) for x in s["ring"].cpu())
    slots, pos, offs, lens_out = [], [], [0], []
    for r, (x, new) in enumerate(zip(s["lens"].tolist(), s["new"].tolist())):
        for p in range(x, x + new):
            if p % P == 0:
                table[r, p // P] = free[head]
                head, count = (head + 1) % N, count - 1
            slots.append(int(table[r, p // P]) * P + p % P)
            pos.append(p)
        offs.append(offs[-1] + new)
        lens_out.append(x + new)
    pad = s["n_slots"] - len(slots)
    for r in s["rows"].tolist():
        for j in range(-(-lens_out[r] // P)):
            free[(head + count) % N] = table[r, j]
            count += 1
    i32 = lambda v: np.asarray(v, dtype=np.int32)  # noqa: E731
    return {"table": table, "slots": i32(slots + [-1] * pad), "pos": i32(pos + [0] * pad), "offs": i32(offs),
            "lens": i32(lens_out), "free": free, "ring": i32([head, count])}


def _exact_rope(case, s):
    rot, T = case["rot"], case["tok"]
    turns, scale = _turns(case)
    ang = s["pos"].double()[:, None, None] * torch.tensor(turns, device="cuda", dtype=torch.float64) * (2 * math.pi)
    z = torch.polar(torch.full_like(ang, scale), ang)            # one complex factor a pair
    pair = (lambda x: (x[..., 0:rot:2], x[..., 1:rot:2])) if case["inter"] else \
        (lambda x: (x[..., :rot // 2], x[..., rot // 2:rot]))

    def forward(x, w):
        if w is not None:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["d"] + EPS) * w
        y = torch.complex(*pair(x)) * z
        out = x.clone()
        if case["inter"]:
            out[..., 0:rot:2], out[..., 1:rot:2] = y.real, y.imag
        else:
            out[..., :rot // 2], out[..., rot // 2:rot] = y.real, y.imag
        return out

    up = lambda x: None if x is None else x.double()  # noqa: E731
    if case["op"] == "rope":
        q, k = forward(up(s["q"]), up(s["wq"])), forward(up(s["k"]), up(s["wk"]))
        if not case["cache"]:
            return {"q": q.cpu().numpy(), "k": k.cpu().numpy()}
        out = {"q": q.cpu().numpy()}
        slot = s["slots"].cpu().numpy()
        for name, x in (("k_cache", k), ("v_cache", s["v"].double())):
            cache, x = s[name].double().cpu().numpy(), x.cpu().numpy()
            for t in range(T):
                if slot[t] >= 0:
                    cache[slot[t] // case["page"], :, slot[t] % case["page"]] = x[t]
            out[name] = cache
        return out
    out = {}
    for name, x, w, dy in (("q", s["q"], s["wq"], s["dy"]), ("k", s["k"], s["wk"], s["dk"])):
        x, w = up(x).clone().requires_grad_(True), up(w)
        ins = [x]
        if w is not None:
            w = w.clone().requires_grad_(True)
            ins.append(w)
        got = torch.autograd.grad((forward(x, w) * dy.double()).sum(), ins)
        out["d" + name] = got[0].cpu().numpy()
        if w is not None:
            out["dw" + name] = got[1].cpu().numpy()
    order = ["dq", "dk", "dwq", "dwk"] if case["norm"] else ["dq", "dk"]
    return {k: out[k] for k in order}


def _exact_attn(case, s):
    n, B, Hq, Hkv, d = (case[k] for k in ("n", "B", "Hq", "Hkv", "d"))
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
        page, at = s["table"][r, j // case["page"]].long(), j % case["page"]
        for h in range(Hkv):
            k, v = s["k_cache"][page, h, at].double(), s["v_cache"][page, h, at].double()
            for g in range(h * G, h * G + G):
                out[r, :, g] = torch.softmax(s["q"][r, :, g].double() @ k.T / math.sqrt(d), -1) @ v
    return out.cpu().numpy()
