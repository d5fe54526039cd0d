"""The 8-bit paged cache in 64 bits, from its definition (include/hybrid_softmax.h), one group of tokens at a
time, and what its tests share."""
import math

import torch

GROUP = 16
F8 = torch.float8_e4m3fn
NAN = 0x7f                      # a code of NaN


def values(codes, scales):
    """Codes [pages, Hkv, P, d] and scales [pages, Hkv, P / 16] as float64 values."""
    return codes.view(torch.uint8).view(F8).double() * scales.double().repeat_interleave(GROUP, 2)[..., None]


def least_scale(amax):
    """2^E, E >= -126 the least with amax <= 448 * 2^E."""
    e = -126
    if amax > 0:
        e = max(-126, math.frexp(amax)[1] - 10)
        while amax > 448.0 * 2.0 ** e:
            e += 1
        while e > -126 and amax <= 448.0 * 2.0 ** (e - 1):
            e -= 1
    return 2.0 ** e


def check_write(before, after, x, slots, loose, what):
    """One head-major cache after a write of x [T, Hkv, d] (float64, what is rounded) to slots, T ints.
    before, after: (codes, scales).  `loose`: how far the kernel's x may be from this one, relative to a row's largest
    entry (0: not at all)."""
    codes0, scales0 = (t.cpu() for t in before)
    codes1, scales1 = (t.cpu() for t in after)
    got, x = values(codes1, scales1), x.cpu()
    pages, Hkv, P, d = codes0.shape
    groups = {}
    for t, slot in enumerate(slots):
        if 0 <= slot < pages * P:
            groups.setdefault(slot // GROUP, []).append(t)
    touched = torch.zeros(pages, P // GROUP, dtype=torch.bool)
    for g, ts in groups.items():
        page, sub = g * GROUP // P, g * GROUP % P // GROUP
        touched[page, sub] = True
        at = [slots[t] % GROUP for t in ts]
        rest = [i for i in range(GROUP) if i not in at]
        new = x[ts].transpose(0, 1)                                     # [Hkv, tokens, d]
        finite = new.isfinite()
        rows = slice(sub * GROUP, sub * GROUP + GROUP)
        c0, c1 = codes0.view(torch.uint8)[page, :, rows], codes1.view(torch.uint8)[page, :, rows]
        fresh = 0 in at
        for h in range(Hkv):
            s = float(scales1[page, h, sub])
            amax = float(torch.where(finite[h], new[h].abs(), 0.0).max())
            low, high = least_scale(amax * (1 - loose)), least_scale(amax * (1 + loose))
            if not fresh:
                low, high = max(low, float(scales0[page, h, sub])), max(high, float(scales0[page, h, sub]))
            assert low <= s <= high and math.frexp(s)[0] == 0.5, (what, "scale", g, h, s, low, high)
            # half a step at the value: 2^-4 of it, and of the subnormals 2^-10 of the scale
            y = torch.where(finite[h], new[h], 0.0)
            far = (got[page, h, rows][at] - y).abs()
            bound = (y.abs() * 2.0 ** -4).clamp(min=s * 2.0 ** -10) * (1 + 2.0 ** -20) + 1.07 * loose * y.abs().amax(-1, keepdim=True)
            assert bool(((far <= bound) | ~finite[h]).all()), (what, "value", g, h)
            assert torch.equal(got[page, h, rows][at].isnan(), ~finite[h]), (what, "infinities", g, h)
            if fresh:
                assert not bool(c1[h][rest].any()), (what, "the rest of a fresh group", g, h)
            elif s == float(scales0[page, h, sub]):
                assert torch.equal(c1[h][rest], c0[h][rest]), (what, "kept", g, h)
            else:
                old = c0[h][rest].view(F8).double() * (float(scales0[page, h, sub]) / s)
                assert torch.equal(c1[h][rest].view(F8).double(), old.float().to(F8).double()), (what, "moved", g, h)
    still = ~touched
    assert torch.equal(scales1.transpose(1, 2)[still], scales0.transpose(1, 2)[still]), (what, "other scales")
    by_group = lambda c: c.view(torch.uint8).view(pages, Hkv, P // GROUP, GROUP, d).transpose(1, 2)[still]  # noqa: E731
    assert torch.equal(by_group(codes1), by_group(codes0)), (what, "other codes")
