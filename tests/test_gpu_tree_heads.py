"""Keys that are not finite in the rotated columns of one head: s[b,i,h,t] reads that head's alone, so that the others
know nothing of them, whichever kernel computes the call.  Oracle and tolerances are those of tests/test_gpu_tree.py."""
from dataclasses import replace

import numpy as np
import pytest

from paper_2503_01586_b200 import inputs as gen

from .test_gpu_tree import call_tree, check_tree, ek, tree_state  # noqa: F401  (ek is a fixture)

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
TWELVE = replace(gen.TINY, n_h=12, d_h=96, r=3, d_c=384, d=1152)      # heads whose columns start on no 16-byte boundary

CASES = {
    # kernel for any shape (few rows; pages of 4)
    "any-shape": (gen.TINY, 0, 5, [60, 33], [5, 2], 0), "any-shape-pages": (gen.LLAMA7B_75, 0, 3, [140, 50], [3, 3], 4),
    # nodes as query rows of the decode kernel
    "rows": (gen.LLAMA7B_75, 0, 4, [500, 131], [4, 3], 0), "rows-slrd": (gen.LLAMA7B_75, 512, 7, [300], [7], 64),
    # dense products: one block holds all rows, pairs, several row blocks, several tiles and pieces
    "dense-block": (gen.TINY, 0, 17, [2600, 40], [17, 9], 16), "dense-odd": (TWELVE, 0, 20, [700, 330], [20, 3], 0),
    "dense-pair": (gen.LLAMA7B_75, 0, 17, [300, 1100], [17, 11], 64), "dense-13b": (gen.LLAMA13B_75, 0, 33, [290], [33], 0),
    "dense-slrd": (gen.LLAMA7B_75, 512, 64, [513, 257], [64, 60], 32), "dense-87.5": (gen.SWEEP_875, 0, 24, [400], [24], 8),
}


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("case", list(CASES))
def test_other_heads_know_nothing_of_it(ek, case, bad):
    """One column or all of one head's, in a committed token of the first, of a middle and of the last tile, and in a
    drafted one that some nodes see."""
    w, d_ck, m, lens, nodes, ps = CASES[case]
    r2 = 2 * w.r
    for k, (head, cols) in enumerate(((1, slice(0, r2)), (w.n_h - 1, slice(r2 - 1, r2)), (w.n_h // 2, slice(0, 1)))):
        s = tree_state(ek, w, lens, nodes, m, ps=ps, seed=k, d_ck=d_ck)
        n, prefix = lens[0], lens[0] - nodes[0]
        at = ((0, prefix - 1), (n // 2,), (prefix + nodes[0] // 2, 17))[k]
        for t in at:
            s["rope"][s["where"][0][t], head * r2:(head + 1) * r2][cols] = bad
        heads = sorted({0, 1, head - 1, head, (head + 1) % w.n_h, w.n_h - 1})
        out = call_tree(ek, s)
        check_tree(s, out, heads)
        others = [h for h in range(w.n_h) if h != head]
        assert out[:, :, others].isfinite().all()


@pytest.mark.parametrize("case", ["dense-block", "dense-odd", "dense-pair", "rows"])
def test_many_of_them(ek, case):
    """Another head's columns in every seventh token, and values that are nobody's alone: a latent, which all heads read."""
    w, d_ck, m, lens, nodes, ps = CASES[case]
    r2 = 2 * w.r
    s = tree_state(ek, w, lens, nodes, m, ps=ps, seed=5, d_ck=d_ck)
    for k, t in enumerate(range(3, lens[0] - nodes[0], 7)):
        head = 2 + k % (w.n_h - 3)                          # heads 0, 1 and the last stay whole
        s["rope"][s["where"][0][t], head * r2 + k % r2] = (NAN, INF, -INF)[k % 3]
    check_tree(s, call_tree(ek, s), [0, 1, 2, w.n_h - 1])
    s["lat"][s["where"][0][lens[0] - nodes[0] - 1], 0] = NAN
    out = call_tree(ek, s)
    assert out[0, :nodes[0]].isnan().all() and out[1].isfinite().all()


def test_a_cache_of_them(ek):
    """All but two heads' columns of all tokens."""
    w, d_ck, m, lens, nodes, ps = CASES["dense-pair"]
    s = tree_state(ek, w, lens, nodes, m, ps=ps, seed=6, d_ck=d_ck)
    for b in range(2):
        s["rope"][s["where"][b], 2 * 2 * w.r:] = NAN
    out = call_tree(ek, s)
    check_tree(s, out, [0, 1])
    for b, k in enumerate(nodes):
        assert out[b, :k, 2:].isnan().all()


@pytest.mark.parametrize("n_h,d_c,lens,m", [(32, 4096, [1100, 700], 32), (16, 8192, [2048, 300], 64)])
def test_wide_latents_and_a_cache_of_them(ek, n_h, d_c, lens, m):
    """Where every score of a tile is computed again over thousands of latents, the waits of the others are long, but run out
    nowhere."""
    w = replace(gen.TINY, n_h=n_h, d_h=128, r=8, d_c=d_c, d=n_h * 128)
    s = tree_state(ek, w, lens, [m, m], m, seed=7)
    for b in range(2):
        s["rope"][s["where"][b], 2 * 2 * w.r:] = NAN
    out = call_tree(ek, s)
    check_tree(s, out, [1], seqs=[1])
    assert out[:, :, :2].isfinite().all() and out[:, :, 2:].isnan().all()
