"""Tree attention in block pairs where the second block has nothing of a unit: sequences whose last tile ends in the first
block's half, last value tiles of a few latents.  Many calls after one another, each with the same bits and no wait that
ran out."""
from dataclasses import replace

import pytest
import torch

from paper_2503_01586_b200 import inputs as gen

from .test_gpu_tree import call_tree, check_tree, ek, i32, tree_state  # noqa: F401  (ek is a fixture)

pytestmark = pytest.mark.gpu

NARROW_END = replace(gen.TINY, n_h=16, d_h=64, r=4, d_c=1032, d=1024)          # 8 latents in the last value tile
NARROW_64 = replace(gen.TINY, n_h=24, d_h=64, r=2, d_c=840, d=1536)            # 72 (two chunks)


@pytest.mark.parametrize("w,d_ck,m,ps", [(gen.LLAMA13B_75, 0, 33, 32), (gen.LLAMA7B_75, 512, 40, 64), (NARROW_END, 0, 20, 0), (NARROW_END, 0, 24, 16),
                                         (NARROW_64, 0, 17, 8), (gen.SWEEP_875, 0, 64, 0)])
def test_the_second_block_has_nothing_of_a_unit(ek, w, d_ck, m, ps):
    lens = [m, m + 1, 257, 300, 384, 513, 640, 1025, 1100, 2305, 2400] * 2
    nodes = [m, 1, m, m // 2, m, m - 1, m, 3, m, m, m // 3] * 2
    s = tree_state(ek, w, lens, nodes, m, ps=ps, seed=m, d_ck=d_ck)
    want = call_tree(ek, s)
    check_tree(s, want, [0, w.n_h - 1], seqs=range(11))
    lens, nodes = i32(lens), i32(nodes)
    for _ in range(100):
        out = ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], lens, nodes, s["mask"], s["ws"])
        assert ek.elitekv_check_status(s["layer"]) == 0
        assert torch.equal(out, want)
