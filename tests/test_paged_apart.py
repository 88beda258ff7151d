"""What a paged call writes lies apart from what it reads and from what else it
writes, buffer by buffer; refused before anything is enqueued, so no GPU is
needed."""
import ctypes

import pytest

import paper_2608_27875_amd as hyq
from test_paged_abi import EINVAL, lib   # noqa: F401 (lib is a fixture)

STEP = 1 << 36
NAMES = ["q", "k", "v", "pos", "q_weight", "k_weight", "inv_freq", "cu", "lens", "table", "new_table", "ws", "out",
         "Q", "K", "V", "keep", "new_lens", "ck", "cv", "cks", "cvs", "mass"]
HEADS, KV, PAGE, PAGES, T, B, MAX_PAGES = 8, 2, 16, 10, 6, 2, 8
BUDGET, NEW_PAGES = 40, 3
POOL = PAGES * KV * PAGE
SIZES = dict(q=T * HEADS * 256, k=T * KV * 256, v=T * KV * 256, pos=T * 4, q_weight=256, k_weight=256, inv_freq=256,
             cu=(B + 1) * 4, lens=B * 4, table=B * MAX_PAGES * 4, new_table=B * NEW_PAGES * 4, ws=1 << 20,
             out=T * HEADS * 512, Q=T * HEADS * 256, K=T * KV * 256, V=T * KV * 256, keep=B * KV * BUDGET * 4,
             new_lens=B * 4, ck=POOL * 128, cv=POOL * 128, cks=POOL * 4, cvs=POOL * 4, mass=POOL * 4)


def places(**moved):
    at = {n: STEP * (i + 1) for i, n in enumerate(NAMES)}
    at.update(moved)
    return at


def call(lib, name, at):   # noqa: F811
    c = hyq._PCache(HEADS, KV, 128, PAGE, PAGES, 8, 0, at["ck"], at["cv"], at["cks"], at["cvs"], at["mass"])
    b = hyq._PBatch(B, T, 4, 100, MAX_PAGES, at["cu"], at["lens"], at["table"])
    r = hyq._Rope(128, 0, 1e-6, at["q_weight"], at["k_weight"], at["inv_freq"])
    rows = [at["q"], HEADS * 128, at["k"], KV * 128, at["v"], KV * 128, at["pos"]]
    if name == "norm_rope":
        return lib.hyq_norm_rope(hyq.Shape(B=2, Hq=HEADS, Hkv=KV, L=3).c(), r, *rows, at["Q"], at["K"], at["V"], None)
    if name == "append":
        return lib.hyq_paged_append(c, b, r, *rows, at["Q"], None)
    if name == "attn":
        return lib.hyq_paged_attn(c, b, at["q"], ctypes.c_float(0.1), hyq.MASS_ADD, at["out"], 0, at["ws"],
                                  ctypes.c_size_t(1 << 20), None)
    return lib.hyq_evict(c, B, at["lens"], at["table"], MAX_PAGES, 100, BUDGET, 4, at["new_table"], NEW_PAGES,
                         at["keep"], at["new_lens"], None)


CALLS = {   # written, read
    "norm_rope": (["Q", "K", "V"], ["q", "k", "v", "pos", "q_weight", "k_weight", "inv_freq"]),
    "append": (["Q", "ck", "cv", "cks", "cvs", "mass"],
               ["q", "k", "v", "pos", "q_weight", "k_weight", "inv_freq", "cu", "lens", "table"]),
    "attn": (["out", "ws", "mass"], ["q", "ck", "cv", "cks", "cvs", "cu", "lens", "table"]),
    "evict": (["keep", "new_lens", "ck", "cv", "cks", "cvs", "mass"], ["lens", "table", "new_table"]),
}
PAIRS = [(n, w, x) for n, (out, ins) in CALLS.items() for i, w in enumerate(out) for x in ins + out[i + 1:]]


@pytest.mark.parametrize("name,written,other", PAIRS)
def test_overlaps_are_refused(lib, name, written, other):   # noqa: F811
    """On top of each other, and by the last 16 bytes of the one before."""
    at = places()
    size = lambda n: {"ws": 16}.get(n, SIZES[n])   # noqa: E731 (whatever is needed of the workspace, its start is)
    for first, second in ((written, other), (other, written)):
        for shift in (0, (size(first) - 1) // 16 * 16):
            assert call(lib, name, places(**{second: at[first] + shift})) == EINVAL, (first, second, shift)
            assert "overlap" in hyq.hyq_last_error()
