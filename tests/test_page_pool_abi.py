"""hybrid_page_append and hybrid_page_release refuse arguments that share memory, on the host."""
import ctypes

import pytest

from paper_2608_06628_gb300 import build as B
from paper_2608_06628_gb300 import hybrid as H

N, SLOTS, PAGES, WIDTH, BASE, APART = 6, 40, 30, 4, 1 << 20, 4096
# argument -> its ints; outputs end with a star ("free" of a release is read and written)
APPEND = {"lens": N, "n_new": N, "free": PAGES, "ring_in": 2, "table*": N * WIDTH, "slots*": SLOTS, "positions*": SLOTS,
          "offsets*": N + 1, "lens_out*": N, "ring_out*": 2}
RELEASE = {"rows": 3, "lens": N, "table": N * WIDTH, "free*": PAGES, "ring_in": 2, "ring_out*": 2}


@pytest.fixture(scope="module")
def L():
    B.build()
    return H.lib()


def call(L, name, at):
    pg = ctypes.byref(H.hybrid_page_cfg(16, PAGES, WIDTH))
    p = {k.rstrip("*"): v for k, v in at.items()}
    if name == "append":
        return L.hybrid_page_append(pg, N, p["lens"], p["n_new"], p["free"], p["ring_in"], p["table"], p["slots"], p["positions"],
                                    SLOTS, p["offsets"], p["lens_out"], p["ring_out"], None)
    return L.hybrid_page_release(pg, N, p["rows"], 3, p["lens"], p["table"], p["free"], p["ring_in"], p["ring_out"], None)


@pytest.mark.parametrize("name,args", [("append", APPEND), ("release", RELEASE)])
def test_outputs_that_share_memory(L, name, args):
    apart = {k: BASE + APART * i for i, k in enumerate(args)}
    for a, n in args.items():
        for b, m in args.items():
            if a == b or not (a.endswith("*") or b.endswith("*")):
                continue
            # the first and the last int of b, from either side
            for shift in (0, 4 * (m - 1), -4 * (n - 1)):
                assert call(L, name, {**apart, a: apart[b] + shift}) == H.HYBRID_ERR_INVALID_ARG, (a, b, shift)
