"""The softmax-layer entry points on the host, without a GPU: argument checks before the device is
touched, workspace sizes, and the rotation's frequencies against the formulas."""
import ctypes
import math

import pytest

import softmax_reference as R
from paper_2608_06628_gb300 import build as B
from paper_2608_06628_gb300 import hybrid as H

OK, BAD, UNSUP = H.HYBRID_OK, H.HYBRID_ERR_INVALID_ARG, H.HYBRID_ERR_UNSUPPORTED
PTR = 1 << 20     # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def L():
    B.build()
    return H.lib()


def cfg(d=128, Hq=16, Hkv=4, Bs=32, dt=H.HYBRID_BF16):
    return H.hybrid_cfg(d, 7, Hq, Hkv, Bs, dt)      # feat_dim is not read


def pg(P=32, n=100, m=10):
    return H.hybrid_page_cfg(P, n, m)


def rope(rot=128, inter=0, scale=1.0, eps=1e-6):
    return H.hybrid_rope_cfg(rot, inter, scale, eps)


# entry point -> (its cases of configuration, argument roles): "p16"/"p8"/"p4" a required pointer, "o16"/"o4"
# one that may be null, "i:<v>" an int or size, "s" the stream.  Pointers differ from one another.
ARGS = {
    "hybrid_page_append": ((pg,), ["i:2", "p4", "p4", "p4", "p4", "p4", "p4", "o4", "i:64", "o4", "p4", "p4", "s"]),
    "hybrid_page_release": ((pg,), ["i:2", "p4", "i:1", "p4", "p4", "p4", "p4", "p4", "s"]),
    "hybrid_qk_norm_rope": ((cfg, rope), ["p16", "i:2048", "p16", "i:512", "i:3", "o16", "o16", "p4", "p8", "p16", "p16", "s"]),
    "hybrid_qk_norm_rope_cache": ((cfg, rope, pg), ["p16", "i:2048", "p16", "i:512", "p16", "i:512", "i:3", "o16", "o16", "p4",
                                                    "p8", "p4", "p16", "p16", "p16", "s"]),
    "hybrid_qk_norm_rope_backward": ((cfg, rope), ["p16", "i:2048", "p16", "i:512", "p16", "p16", "i:3", "p16", "p16", "p4", "p8",
                                                   "p16", "i:100000000", "p16", "p16", "p4", "p4", "s"]),
    "hybrid_paged_attn": ((cfg, pg), ["p16", "p16", "p16", "p4", "p4", "i:2", "i:0", "i:0", "p16", "p16", "i:1000000000", "s"]),
}


def call(L, name, make=None, override=None):
    cfgs, roles = ARGS[name]
    made = [(make or {}).get(f, f)() for f in cfgs]
    args = []
    for i, r in enumerate(roles):
        if override and i in override:
            args.append(override[i])
        elif r == "s":
            args.append(None)
        elif r.startswith("i:"):
            args.append(int(r[2:]))
        else:
            args.append(PTR + 4096 * i)
    return getattr(L, name)(*[ctypes.byref(m) if m is not None else None for m in made], *args)


@pytest.mark.parametrize("name", sorted(ARGS))
def test_every_pointer_is_checked_on_the_host(L, name):
    cfgs, roles = ARGS[name]
    assert len(cfgs) + len(roles) == len(getattr(L, name).argtypes)
    for i, r in enumerate(roles):
        if r[0] not in "po":
            continue
        align, at = int(r[1:]), PTR + 4096 * i
        assert call(L, name, override={i: at + align // 2}) == BAD, (name, i, "misaligned")
        if r[0] == "p":
            assert call(L, name, override={i: None}) == BAD, (name, i, "null")
    for k, f in enumerate(cfgs):
        assert call(L, name, {f: lambda: None}) == BAD, (name, k)


@pytest.mark.parametrize("name", [n for n in sorted(ARGS) if cfg in ARGS[n][0]])
@pytest.mark.parametrize("bad,code", [(dict(d=96), UNSUP), (dict(dt=7), UNSUP), (dict(Hq=257, Hkv=257), UNSUP),
                                      (dict(Hq=6, Hkv=4), BAD), (dict(Hq=4, Hkv=8), BAD), (dict(Hkv=0), UNSUP)])
def test_configurations_outside_the_set(L, name, bad, code):
    assert call(L, name, {cfg: lambda: cfg(**bad)}) == code


@pytest.mark.parametrize("name", [n for n in sorted(ARGS) if pg in ARGS[n][0]])
@pytest.mark.parametrize("bad,code", [(dict(P=24), UNSUP), (dict(P=256), UNSUP), (dict(P=0), UNSUP), (dict(n=0), BAD),
                                      (dict(m=0), BAD), (dict(n=-1), BAD), (dict(n=2 ** 26), UNSUP), (dict(m=2 ** 26), UNSUP)])
def test_page_configurations_outside_the_set(L, name, bad, code):
    assert call(L, name, {pg: lambda: pg(**bad)}) == code


@pytest.mark.parametrize("name", [n for n in sorted(ARGS) if rope in ARGS[n][0]])
@pytest.mark.parametrize("bad,code", [(dict(rot=144), UNSUP), (dict(rot=24), UNSUP), (dict(rot=-16), UNSUP), (dict(inter=2), BAD),
                                      (dict(eps=-1.0), BAD), (dict(eps=math.nan), BAD), (dict(scale=math.inf), BAD)])
def test_rotations_outside_the_set(L, name, bad, code):
    assert call(L, name, {rope: lambda: rope(**bad)}) == code


def test_numbers_out_of_range(L):
    a, r, c, k, b, t = ("hybrid_page_append", "hybrid_page_release", "hybrid_qk_norm_rope_cache", "hybrid_qk_norm_rope",
                        "hybrid_qk_norm_rope_backward", "hybrid_paged_attn")
    for name, over, code in [
        (a, {0: -1}, BAD), (a, {0: 65537}, UNSUP), (a, {8: -1}, BAD), (r, {0: -1}, BAD), (r, {2: -1}, BAD), (r, {2: 65537}, UNSUP),
        (a, {11: PTR + 4096 * 4}, BAD),                 # ring_out is ring_in
        (a, {10: PTR + 4096 * 1}, BAD),                 # lens_out is lens
        (r, {7: PTR + 4096 * 6}, BAD),
        (k, {4: -1}, BAD), (k, {1: 2047}, BAD), (k, {1: 2040}, BAD), (k, {1: 2052}, BAD), (k, {3: 504}, BAD),
        (k, {9: PTR, 1: 4096}, BAD),                    # in place on a strided input
        (k, {10: PTR + 4096 * 2, 3: 1024}, BAD), (c, {12: PTR, 1: 4096}, BAD),
        (c, {5: 504}, BAD), (c, {5: 515}, BAD), (c, {6: -1}, BAD),
        (b, {6: -1}, BAD), (b, {12: 100}, BAD), (b, {15: None}, BAD), (b, {7: None}, BAD),
        (t, {5: -1}, BAD), (t, {5: 65537}, UNSUP), (t, {6: -1}, BAD), (t, {7: -1}, BAD), (t, {10: 100}, BAD),
    ]:
        assert call(L, name, override=over) == code, (name, over)
    for Bs in (0, 129):
        assert call(L, t, {cfg: lambda Bs=Bs: cfg(Bs=Bs)}) == UNSUP


def test_nothing_to_do(L):
    """No requests or tokens: pointers may be null, configurations are still checked."""
    for name, count in (("hybrid_paged_attn", 5), ("hybrid_qk_norm_rope", 4), ("hybrid_qk_norm_rope_cache", 6)):
        over = {i: None for i, r in enumerate(ARGS[name][1]) if r[0] in "po"}
        over[count] = 0
        assert call(L, name, override=over) == OK
        assert call(L, name, {cfg: lambda: cfg(d=96)}, over) == UNSUP
    over = {i: None for i, r in enumerate(ARGS["hybrid_page_append"][1]) if r[0] in "po"}
    assert call(L, "hybrid_page_append", override={**over, 0: 0, 8: 0}) == OK
    over = {i: None for i, r in enumerate(ARGS["hybrid_page_release"][1]) if r[0] in "po"}
    assert call(L, "hybrid_page_release", override={**over, 2: 0}) == OK


def test_workspace_sizes(L):
    assert H.hybrid_paged_attn_workspace_bytes(cfg(), pg(), 3) > 0
    assert H.hybrid_qk_norm_rope_workspace_bytes(cfg(), 3) > 0
    for bad in (dict(d=96), dict(Bs=0), dict(Bs=129), dict(dt=5)):
        assert H.hybrid_paged_attn_workspace_bytes(cfg(**bad), pg(), 3) == 0
    assert H.hybrid_paged_attn_workspace_bytes(cfg(), pg(P=24), 3) == 0
    assert H.hybrid_paged_attn_workspace_bytes(cfg(), pg(), -1) == 0
    assert H.hybrid_qk_norm_rope_workspace_bytes(cfg(d=96), 3) == 0
    assert H.hybrid_qk_norm_rope_workspace_bytes(cfg(), -1) == 0


@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("kind,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("yarn", 16.0), ("yarn", 1.0)])
@pytest.mark.parametrize("base", [10000.0, 500000.0])
def test_frequencies(L, rot, kind, factor, base):
    """64-bit fractions of a turn: 2^-52 of the frequency, from double arithmetic (pow within 2 ulp, three
    more operations), and 2^-64 from the fraction."""
    code = {"none": H.HYBRID_ROPE_NONE, "linear": H.HYBRID_ROPE_LINEAR, "ntk": H.HYBRID_ROPE_NTK, "yarn": H.HYBRID_ROPE_YARN}
    rc, freqs = H.make_rope(rot, True, base=base, kind=code[kind], factor=factor, orig_len=2048.0, device="cpu")
    want, scale = R.turns(rot, kind, base, factor, 2048.0)
    assert (rc.rot_dim, rc.interleaved) == (rot, 1) and abs(rc.scale - scale) <= 2 ** -23
    assert len(freqs) == rot // 2
    for f, t in zip(freqs.tolist(), want):
        assert f > 0 and abs(f / 2.0 ** 64 - t) <= 2.0 ** -48 * t + 2.0 ** -64


def test_frequencies_refused(L):
    arr, scale = (ctypes.c_ulonglong * 64)(), ctypes.c_float()

    def freqs(kind=0, base=1e4, factor=2.0, orig=4096.0, fast=32.0, slow=1.0, rot=64):
        sc = H.hybrid_rope_scaling(kind, base, factor, orig, fast, slow)
        return H.hybrid_rope_freqs(sc, rot, arr, scale, check=False)

    assert freqs() == OK and freqs(3) == OK
    assert freqs(rot=24) == UNSUP and freqs(rot=0) == UNSUP and freqs(rot=144) == UNSUP and freqs(4) == UNSUP and freqs(-1) == UNSUP
    for bad in (dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(kind=1, factor=0.5), dict(kind=2, factor=math.nan),
                dict(kind=3, orig=0.0), dict(kind=3, fast=1.0), dict(kind=3, slow=-1.0), dict(kind=3, fast=math.inf)):
        assert freqs(**bad) == BAD, bad
    assert L.hybrid_rope_freqs(None, 64, arr, ctypes.byref(scale)) == BAD
