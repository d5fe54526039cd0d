"""Plain implementations of the softmax-layer operators in 64 bits, written from their definitions
(include/hybrid_softmax.h). They run on whatever device their inputs are on."""
import math

import torch


def turns(rot, kind="none", base=10000.0, factor=1.0, orig=4096.0, fast=32.0, slow=1.0):
    """Turns per position of each pair, and the factor on cosine and sine."""
    if kind == "ntk":
        base = base * factor ** (rot / (rot - 2))
    out = []
    for i in range(rot // 2):
        t = base ** (-2.0 * i / rot) / (2 * math.pi)
        if kind == "linear":
            t /= factor
        if kind == "yarn":
            g = min(1.0, max(0.0, (orig * t - slow) / (fast - slow)))
            t = t / factor * (1 - g) + t * g
        out.append(t)
    return out, (0.1 * math.log(factor) + 1 if kind == "yarn" else 1.0)


def norm_rotate(x, w, pos, t, scale, inter, eps):
    """x [T, H, d] float64 -> normalised (w not None) and rotated."""
    if w is not None:
        x = x * ((x * x).mean(-1, keepdim=True) + eps).rsqrt() * w
    rot = 2 * len(t)
    if rot == 0:
        return x
    # reduce to a fraction of a turn first, exactly in integers where the position is large
    t = torch.tensor(t, dtype=torch.float64, device=x.device)
    ang = 2 * math.pi * torch.remainder(pos.double()[:, None, None] * t, 1.0)
    c, s = torch.cos(ang) * scale, torch.sin(ang) * scale
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., :rot // 2], x[..., rot // 2:rot])
    y0, y1 = a * c - b * s, b * c + a * s
    y = torch.stack([y0, y1], -1).flatten(-2) if inter else torch.cat([y0, y1], -1)
    return torch.cat([y, x[..., rot:]], -1)


def norm_rotate_grad(x, w, dy, pos, t, scale, inter, eps):
    """Gradients of sum(dy * norm_rotate(x, w)) by the formula, and sum |terms| of dw."""
    rot, d = 2 * len(t), x.shape[-1]
    dn = norm_rotate(dy, None, -pos.long(), t, scale, inter, eps)        # R^T: the rotation by -t
    assert dn.shape == dy.shape and rot <= d
    if w is None:
        return dn, None, None
    r = ((x * x).mean(-1, keepdim=True) + eps).rsqrt()
    xh, u = x * r, dn * w
    return r * (u - xh * (u * xh).mean(-1, keepdim=True)), (dn * xh).sum((0, 1)), (dn * xh).abs().sum((0, 1))


def visible(length, window, sink):
    if window == 0:
        return list(range(length))
    lo = max(0, length - window)
    return list(range(min(sink, lo))) + list(range(lo, length))


def paged_attention(q, k_cache, v_cache, table, lens, window, sink):
    """q [n, B, Hq, d]; caches [pages, Hkv, P, d] -> [n, B, Hq, d] float64."""
    n, B, Hq, d = q.shape
    Hkv, P = k_cache.shape[1], k_cache.shape[2]
    G = Hq // Hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    for r in range(n):
        j = visible(int(lens[r]), window, sink)
        if not j:
            continue
        j = torch.tensor(j, device=q.device)
        page, at = table[r][j // P].long(), j % P
        k, v = k_cache[page, :, at].double(), v_cache[page, :, at].double()      # [keys, Hkv, d]
        qr = q[r].double().view(B, Hkv, G, d)
        x = torch.einsum("bhgd,khd->bhgk", qr, k) / math.sqrt(d)
        out[r] = torch.einsum("bhgk,khd->bhgd", torch.softmax(x, -1), v).reshape(B, Hq, d)
    return out


class Pool:
    """The page pool's rules one request at a time (lists of ints)."""

    def __init__(self, P, n_pages, max_pages, free, head, count, table):
        self.P, self.N, self.max_pages = P, n_pages, max_pages
        self.free, self.head, self.count, self.table = list(free), head, count, [list(r) for r in table]

    def append(self, lens, new, n_slots):
        slots, pos, offs, out = [-1] * n_slots, [0] * n_slots, [0], []
        at, asked, taken, bad = 0, 0, 0, False
        for r, (x, y) in enumerate(zip(lens, new)):
            tok, end = max(y, 0), x + y
            ok = x >= 0 and y >= 0 and end <= self.max_pages * self.P
            need = -(-end // self.P) - -(-x // self.P) if ok else 0
            served = ok and (need == 0 or asked + need <= self.count) and at + tok <= n_slots
            if served:
                old = -(-x // self.P)
                for j in range(old, -(-end // self.P)):
                    self.table[r][j] = self.free[(self.head + asked + j - old) % self.N]
                for i in range(y):
                    p = x + i
                    slots[at + i], pos[at + i] = self.table[r][p // self.P] * self.P + p % self.P, p
                taken = max(taken, asked + need) if need else taken
            bad |= not served
            out.append(end if served else x)
            at, asked = at + tok, asked + need
            offs.append(min(at, n_slots))
        self.head, self.count = (self.head + taken) % self.N, self.count - taken
        return slots, pos, offs, out, bad

    def release(self, rows, lens):
        for r in rows:
            for j in range(-(-lens[r] // self.P)):
                self.free[(self.head + self.count) % self.N] = self.table[r][j]
                self.count += 1
