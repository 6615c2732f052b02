"""The oracle of tree decoding against hand-worked cases and the oracle of the causal rule, and the refusals of the entry
points that need no device (nothing is launched)."""
import ctypes as C

import numpy as np
import pytest

from oracle import elitekv_oracle as O
from oracle import tree_oracle as T


def test_masks_of_a_hand_drawn_tree():
    #   0 - 1 - 3
    #    \- 2 - 4 - 5      6 hangs on the committed tokens, 7 names a node that is not before it
    parent = [-1, 0, 0, 1, 2, 4, -1, 9]
    assert T.mask_bits(parent, 8) == [0b1, 0b11, 0b101, 0b1011, 0b10101, 0b110101, 0b1000000, 0b10000000]
    assert T.mask_bits(None, 4) == [1, 3, 7, 15]


def test_tables_by_hand():
    # pages of 4: sequence 0 holds 3 tokens in page 9 and gets 2 (one fits, one opens page 7, the top of the stack),
    # sequence 1 holds 4 in page 2, keeps page 5 from an earlier step, gets 1; sequence 2 is empty and gets 5 (pages 1, 0)
    out = T.step_tables([3, 4, 0], [2, 1, 5], m=0, n_slots=9, page_table=[[9, -1], [2, 5], [-1, -1]], page_size=4,
                        pages_held=[1, 2, 0], free_pages=[3, 0, 1, 7])
    assert out["slot"] == [39, 28, 20, 4, 5, 6, 7, 0, -1]
    assert out["pos"] == [3, 4, 4, 0, 1, 2, 3, 4, 0] and out["seq_id"] == [0, 0, 1, 2, 2, 2, 2, 2, -1]
    assert out["page_table"].tolist() == [[9, 7], [2, 5], [1, 0]] and out["n_free"] == 1
    assert out["pages_held"] == [2, 2, 2] and out["first"] == [0, 2, 3, 8] and out["result"] == [0, 8, 3, 0]


def test_acceptance_by_hand():
    parent = [-1, 0, 0, 1, 2, 2, -1]
    draft = [5, 8, 8, 1, 3, 4, 5]
    # node 0 and node 6 both draft the right first token, nodes 1 and 2 the right second one: the lowest is followed
    assert T.accept(parent, draft, 5, [8, 1, 3, 77, 0, 0, 0], 7) == ([0, 1, 3], 77)
    assert T.accept(parent, draft, 4, [8, 1, 3, 77, 0, 0, 0], 7) == ([], 4)
    assert T.accept(parent, draft, 5, [8, 2, 3, 77, 0, 0, 0], 7) == ([0, 1], 2)
    assert T.accept(None, [5, 6, 7], 5, [6, 7, 9], 2) == ([0, 1], 7)        # a chain of two nodes, the third is padding


def test_chain_is_the_causal_rule():
    rng = np.random.default_rng(3)
    n_h, d_h, r, d_c, n, m = 3, 8, 2, 6, 9, 4
    idx = np.stack([rng.permutation(d_h // 2)[:r] for _ in range(n_h)])
    q, k_rope, c = rng.standard_normal((m, n_h, d_h)), rng.standard_normal((n, n_h, 2 * r)), rng.standard_normal((n, d_c))
    W_uk, W_uv = rng.standard_normal((d_c, n_h * (d_h - 2 * r))), rng.standard_normal((d_c, n_h * d_h))
    q_pos = n - m + np.arange(m)
    want = O.attend_causal(q, q_pos, k_rope, np.arange(n), c, W_uk, W_uv, idx, d_h)
    parts = [O.absorb_query(q[i], int(q_pos[i]), idx, W_uk, d_h) for i in range(m)]
    got = T.attend_tree(np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts]), k_rope, c, c, W_uv, n - m,
                        T.mask_bits(None, m), d_h ** -0.5)
    np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-12)


def test_unseen_tokens_do_not_touch_a_row():
    rng = np.random.default_rng(4)
    q_rope, q_abs, k_rope, c = (rng.standard_normal(s) for s in ((2, 1, 2), (2, 1, 3), (4, 1, 2), (4, 3)))
    W = rng.standard_normal((3, 4))
    c[3] = np.nan
    out = T.attend_tree(q_rope, q_abs, k_rope, c, c, W, 2, [0b01, 0b10], 1.0)
    assert np.isfinite(out[0]).all() and np.isnan(out[1]).all()
    assert not T.attend_tree(q_rope, q_abs, k_rope[2:], c[2:], c[2:], W, 0, [0, 0], 1.0).any()


# ------------------------------------------------------------------------------- refusals
@pytest.fixture(scope="module")
def ek():
    from paper_2503_01586_b200 import binding, build
    build.build()
    binding.lib()
    return binding


def _cache(ek, paged):
    d = ek.CacheDesc()
    d.rope = d.latent = 1 << 20
    d.n_seqs, d.max_ctx, d.page_size = 4, 100, 16
    if paged:
        d.page_table, d.max_pages_per_seq, d.num_pages = 1 << 21, 8, 40
    return d


def _tables(ek, paged, m):
    t = ek.TablesDesc()
    for i, (name, _) in enumerate(t._fields_):
        setattr(t, name, (1 << 22) + 4096 * i)
    if paged:
        t.page_table = 1 << 21
    if m == 0:
        t.parent = t.tree_mask = None
    return t


@pytest.mark.parametrize("paged", [False, True])
def test_tables_refuse(ek, paged):
    call = ek.lib().elitekv_step_tables

    def refused(cache=None, tables=None, B=2, m=8, n_slots=16, code=ek.ERR_INVALID_ARG):
        cache = cache or _cache(ek, paged)
        tables = tables or _tables(ek, paged, m)
        assert call(C.byref(cache), C.byref(tables), B, m, n_slots, None) == code

    assert call(None, C.byref(_tables(ek, paged, 8)), 2, 8, 16, None) == ek.ERR_INVALID_ARG
    assert call(C.byref(_cache(ek, paged)), None, 2, 8, 16, None) == ek.ERR_INVALID_ARG
    for bad in ({"B": 0}, {"B": 5, "n_slots": 40}, {"m": -1}, {"m": 65, "n_slots": 130}, {"n_slots": 15}, {"n_slots": -1, "m": 0}):
        refused(**bad)
    wide = _cache(ek, paged)
    wide.n_seqs = 10000
    refused(cache=wide, B=8193, m=0, n_slots=5, code=ek.ERR_UNSUPPORTED_SHAPE)
    names = ["held", "fresh", "seq_lens", "first", "seq_id", "pos", "slot", "tree_mask", "result"]
    if paged:
        names += ["page_table", "pages_held", "free_pages", "n_free", "pages_held_out", "n_free_out"]
    for name in names:
        t = _tables(ek, paged, 8)
        setattr(t, name, None)
        refused(tables=t)
    same = [("seq_lens", "held"), ("seq_lens", "fresh")] + ([("pages_held_out", "pages_held"), ("n_free_out", "n_free")] if paged else [])
    for a, b in same:              # every block reads the input while one writes the output
        t = _tables(ek, paged, 8)
        setattr(t, a, getattr(t, b))
        refused(tables=t)
    t = _tables(ek, paged, 0)
    t.parent = 1 << 23             # packed tokens are chains
    refused(tables=t, m=0)
    t = _tables(ek, paged, 8)
    t.slot = t.slot + 4            # 64-bit entries on 8 bytes
    refused(tables=t)
    if paged:
        t = _tables(ek, paged, 8)
        t.page_table = 1 << 24     # not the cache's own table
        refused(tables=t)
        c = _cache(ek, True)
        c.page_size = 24           # not a power of two
        refused(cache=c)


def test_layer_calls_refuse_without_a_layer(ek):
    L, c, p = ek.lib(), _cache(ek, False), 1 << 22
    n = C.c_size_t()
    assert L.elitekv_attend_tree_workspace_size(None, 1, 1, C.byref(n)) == ek.ERR_INVALID_ARG
    assert L.elitekv_attend_tree(None, C.byref(c), p, p, p, p, p, 1, 1, p, 1 << 30, p, None) == ek.ERR_INVALID_ARG
    assert L.elitekv_accept_tree(None, C.byref(c), p, p, p, p, p, p, 1, 1, p, p, p, p, None) == ek.ERR_INVALID_ARG
    assert L.elitekv_append_slots(None, C.byref(c), p, p, p, p, 1, None) == ek.ERR_INVALID_ARG
    assert b"pages" in L.elitekv_strerror(ek.ERR_NO_PAGES)


def test_descriptor_matches_the_header(tmp_path):
    import os
    import subprocess
    from paper_2503_01586_b200 import binding
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [f[0] for f in binding.TablesDesc._fields_]
    src = tmp_path / "t.c"
    src.write_text("\n".join(['#include <stdio.h>', '#include <stddef.h>', '#include "elitekv.h"', 'int main(void){',
                              'printf("%zu\\n", sizeof(elitekv_tables));'] +
                             [f'printf("%zu\\n", offsetof(elitekv_tables, {f}));' for f in names] + ['return 0;}']))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(binding.TablesDesc)] + [getattr(binding.TablesDesc, f).offset for f in names]


def test_tables_of_the_binding_check_sizes():
    import torch
    from paper_2503_01586_b200 import binding
    z = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(AssertionError):
        binding.make_tables(3, 9, 3, z, z)            # host tensors
