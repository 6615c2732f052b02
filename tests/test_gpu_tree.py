"""GPU parity of decoding with a tree of drafted tokens: tables of a step, append by slots, attention of the tree, greedy
acceptance, and the four of them in a row.

Tolerance of the attention, against the float64 oracle on the same bf16 inputs: the probabilities are rounded to bf16 once
(each off by at most 2^-8 of itself) and so is the output (2^-8); sums are fp32.  In the 2-norm over a case each rounding
adds at most its own bound, so 2 x 2^-8 relative, and per element 2 x 2^-8 of what the row could sum to (its largest
magnitude stands in for that, with a factor 4 for cancellation)."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import elitekv_oracle as O
from oracle import tree_oracle as T
from paper_2503_01586_b200 import inputs as gen

from . import harness as H

pytestmark = pytest.mark.gpu

TOL = 2 * 2.0 ** -8


@pytest.fixture(scope="module")
def ek():
    from paper_2503_01586_b200 import binding
    binding.lib()
    return binding


def i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).cuda()


def random_parents(rng, B, m):
    p = np.full((B, m), -1, dtype=np.int32)
    for i in range(1, m):
        p[:, i] = rng.integers(-1 if i % 5 == 0 else 0, i, B)
    return p


# ------------------------------------------------------------------------------- tables
def run_tables(ek, held, fresh, *, m, n_slots, parent=None, table=None, ps=64, pages_held=None, free=None, n_pages=1, max_ctx=0, n_free=None):
    B = len(held)
    plane = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    dev_table = i32(table) if table is not None else None
    cache = ek.make_cache(plane, plane, n_seqs=B, max_ctx=max_ctx, page_table=dev_table, page_size=ps)
    if table is not None:
        cache.num_pages = n_pages
    t = ek.make_tables(B, n_slots, m, i32(held), i32(fresh), parent=i32(parent) if parent is not None else None, page_table=dev_table,
                       pages_held=i32(pages_held) if table is not None else None,
                       free_pages=i32(free if len(free) else [0]) if table is not None else None,
                       n_free=i32([len(free) if n_free is None else n_free]) if table is not None else None)
    ek.elitekv_step_tables(cache, t)
    torch.cuda.synchronize()
    return t, dev_table


def check_tables(t, dev_table, want):
    for k in ("seq_id", "pos", "slot", "seq_lens", "first", "result"):
        assert getattr(t, k).tolist() == list(want[k]), k
    if "tree_mask" in want:
        assert np.array_equal(t.tree_mask.cpu().numpy().view(np.uint64), want["tree_mask"])
    if dev_table is not None:
        assert np.array_equal(dev_table.cpu().numpy(), want["page_table"])
        assert t.pages_held_out.tolist() == want["pages_held"] and t.n_free_out.tolist() == [want["n_free"]]


def paged_state(rng, held, fresh, ps, spare=2):
    pages = [-(-h // ps) + int(rng.random() < 0.4) for h in held]
    width = max(max(p, -(-(h + f) // ps)) for p, h, f in zip(pages, held, fresh)) + 1
    need = sum(max(0, -(-(h + f) // ps) - p) for p, h, f in zip(pages, held, fresh))
    n_pages = sum(pages) + need + spare
    perm = rng.permutation(n_pages)
    table = np.full((len(held), width), -1, dtype=np.int32)
    at = 0
    for b, k in enumerate(pages):
        table[b, :k] = perm[at:at + k]
        at += k
    return pages, table, perm[at:].tolist(), n_pages


@pytest.mark.parametrize("B,most,m,ps", [(1, 1, 1, 64), (1, 7, 7, 16), (5, 33, 33, 1), (300, 64, 64, 8), (17, 16, 16, 64), (1, 1, 0, 64),
                                         (3, 500, 0, 32), (257, 90, 0, 16), (2, 5000, 0, 4), (1000, 3, 0, 128)])
def test_tables(ek, B, most, m, ps):
    rng = np.random.default_rng(B * 1000 + most)
    held, fresh = rng.integers(0, 200, B).tolist(), rng.integers(0, most + 1, B).tolist()
    held[0] = 0
    fresh[B // 2] = most
    parent = random_parents(rng, B, m) if m else None
    n_slots = B * m if m else sum(fresh) + 5
    pages, table, free, n_pages = paged_state(rng, held, fresh, ps)
    t, dev = run_tables(ek, held, fresh, m=m, n_slots=n_slots, parent=parent, table=table, ps=ps, pages_held=pages, free=free, n_pages=n_pages)
    check_tables(t, dev, T.step_tables(held, fresh, m=m, n_slots=n_slots, parent=parent, page_table=table, page_size=ps, pages_held=pages, free_pages=free))
    # contiguous planes, and no parents: chains
    t, dev = run_tables(ek, held, fresh, m=m, n_slots=n_slots, max_ctx=200 + most)
    check_tables(t, dev, T.step_tables(held, fresh, m=m, n_slots=n_slots, max_ctx=200 + most))


def test_tables_of_odd_trees(ek):
    """A chain of 64, roots only, parents that are not before their node, nothing new at all."""
    m = 64
    parent = np.stack([np.arange(m) - 1, np.full(m, -1), np.arange(m), np.full(m, 1 << 20), np.arange(m) - 1])
    held, fresh = [5, 0, 1, 2, 3], [64, 64, 64, 63, 0]
    t, dev = run_tables(ek, held, fresh, m=m, n_slots=5 * m, parent=parent, max_ctx=100)
    check_tables(t, dev, T.step_tables(held, fresh, m=m, n_slots=5 * m, parent=parent, max_ctx=100))


def test_tables_beyond_32_bits_of_rows(ek):
    """Page ids whose rows pass 2^31."""
    table = np.array([[3, 1 << 25, -1]], dtype=np.int32)
    t, dev = run_tables(ek, [130], [70], m=0, n_slots=70, table=table, ps=128, pages_held=[2], free=[], n_pages=(1 << 25) + 1)
    assert t.slot.tolist() == [(1 << 32) + 2 + i for i in range(70)] and t.result.tolist() == [0, 70, 0, 0]


@pytest.mark.parametrize("m", [0, 4])
def test_tables_grant_all_or_nothing(ek, m):
    held, fresh, table = [3, 8], [4, 3], np.array([[2, -1, -1], [5, 1, -1]], dtype=np.int32)
    n_slots = 8

    def nothing(code, detail, **change):
        case = {"held": held, "fresh": fresh, "table": table, "free": [7, 6, 4], "n_pages": 8, "n_slots": n_slots, "pages_held": [1, 2]} | change
        t, dev = run_tables(ek, case["held"], case["fresh"], m=m, n_slots=case["n_slots"], table=case["table"], ps=4,
                            pages_held=case["pages_held"], free=case["free"], n_pages=case["n_pages"], n_free=case.get("n_free"))
        assert t.result.tolist() == [code, 0, 0, detail]
        assert np.array_equal(dev.cpu().numpy(), case["table"])
        assert t.slot.tolist() == [-1] * case["n_slots"] and t.seq_id.tolist() == [-1] * case["n_slots"] and not t.pos.any()
        assert t.seq_lens.tolist() == case["held"] and t.first.tolist() == [0, 0, 0]
        assert t.pages_held_out.tolist() == case["pages_held"]
        assert t.n_free_out.tolist() == [case.get("n_free", len(case["free"]))]

    nothing(ek.ERR_NO_PAGES, 2, free=[])
    nothing(ek.ERR_NO_PAGES, 1, free=[7])
    nothing(ek.ERR_BAD_POSITION, 0, held=[-1, 8])
    nothing(ek.ERR_BAD_POSITION, 1, fresh=[4, -3])
    nothing(ek.ERR_BAD_POSITION, 1, held=[3, 10])                 # more than three pages hold
    nothing(ek.ERR_BAD_POSITION, 0, held=[9, 8])                  # more tokens than pages held
    nothing(ek.ERR_BAD_POSITION, 1, pages_held=[1, 4])            # more pages than the table has
    nothing(ek.ERR_BAD_PAGE, 9, free=[7, 9, 4])                   # one that the step would take
    nothing(ek.ERR_BAD_PAGE, 9, n_free=9)
    nothing(ek.ERR_BAD_PAGE, -1, table=np.array([[-7, -1, -1], [5, 1, -1]], dtype=np.int32))
    if m == 0:
        nothing(ek.ERR_BAD_POSITION, -1, n_slots=6)
    else:
        nothing(ek.ERR_BAD_POSITION, 0, fresh=[5, 1])
    # a bad id that the step does not reach, and the same step with what it needs
    t, dev = run_tables(ek, held, fresh, m=m, n_slots=n_slots, table=table, ps=4, pages_held=[1, 2], free=[99, 6, 4], n_pages=8)
    check_tables(t, dev, T.step_tables(held, fresh, m=m, n_slots=n_slots, page_table=table, page_size=4, pages_held=[1, 2], free_pages=[99, 6, 4]))


# ------------------------------------------------------------------------------- append
@pytest.mark.parametrize("w,T_", [(gen.LLAMA7B_75, 37), (gen.LLAMA7B_75, 2500), (gen.TINY, 50), (replace(gen.TINY, n_h=3, r=3, d_c=40), 21),
                                  (replace(gen.TINY, n_h=3, r=1, d_c=24), 2100)])
def test_append_by_slots(ek, w, T_):
    """The rotation's bits are a pure function of the table, as in elitekv_append; padding and every other row stay as
    they were."""
    st = H.setup(gen.shrink(w, B=1, ctx=T_), lens=[T_])
    rng = np.random.default_rng(T_)
    rows = 2 * T_ + 9
    slot = rng.permutation(rows)[:T_].astype(np.int64)
    pos = rng.integers(0, T_, T_).astype(np.int32)               # siblings share positions
    pad = rng.random(T_) < 0.2
    rope_w = w.n_h * 2 * w.r
    rope, lat = (torch.full((rows, k), -7.0, dtype=torch.bfloat16, device="cuda") for k in (rope_w, w.d_c))
    cache = ek.make_cache(rope, lat, n_seqs=1, max_ctx=rows)
    ek.elitekv_append_slots(st.layer, cache, st.k_e, st.c, torch.from_numpy(np.where(pad, -1 - slot, slot)).cuda(), i32(pos))
    assert ek.elitekv_check_status(st.layer) == 0
    # the rotation of elitekv_append: every product and sum rounded by itself, then once to bf16
    want_rope, want_lat = torch.full_like(rope, -7.0), torch.full_like(lat, -7.0)
    tab = torch.from_numpy(O.rope_table_f32(T_ + 2, w.d_h)).cuda()
    keep = torch.from_numpy(np.flatnonzero(~pad)).cuda()
    x, y = st.k_e[keep].float().view(-1, w.n_h, w.r, 2).unbind(-1)
    cs = tab[torch.from_numpy(pos).cuda()[keep].long()][:, st.idx.cuda().long()]
    rot = torch.stack([x * cs[..., 0] - y * cs[..., 1], x * cs[..., 1] + y * cs[..., 0]], -1).to(torch.bfloat16)
    at = torch.from_numpy(slot).cuda()[keep]
    want_rope[at], want_lat[at] = rot.view(-1, rope_w), st.c[keep]
    assert torch.equal(rope, want_rope) and torch.equal(lat, want_lat)


@pytest.mark.parametrize("T_", [6, 2100])
def test_append_by_slots_records_bad_entries(ek, T_):
    w = gen.LLAMA7B_75
    st = H.setup(gen.shrink(w, B=1, ctx=T_), lens=[T_])
    lat, rope = torch.zeros((T_, w.d_c), dtype=torch.bfloat16, device="cuda"), torch.zeros((T_, 512), dtype=torch.bfloat16, device="cuda")
    cache = ek.make_cache(rope, lat, n_seqs=1, max_ctx=T_)
    for t, slot, pos, detail in ((3, T_, 3, 3), (4, 1 << 40, 4, 4), (2, 2, -1, -1), (1, 1, T_ + 2, T_ + 2)):
        s, p = torch.arange(T_, device="cuda"), torch.arange(T_, dtype=torch.int32, device="cuda")
        s[t], p[t] = slot, pos
        lat.zero_()
        ek.elitekv_append_slots(st.layer, cache, st.k_e, st.c, s, p)
        assert ek.elitekv_check_status(st.layer) == ek.ERR_BAD_POSITION
        assert ek.elitekv_last_status_detail(st.layer) == (t, detail, 1)
        ok = torch.arange(T_, device="cuda") != t
        assert torch.equal(lat[ok], st.c[ok]) and not lat[t].any()


# ------------------------------------------------------------------------------- attention
def tree_state(ek, w, lens, nodes, m, *, ps=0, seed=0, d_ck=0, scale_q=1.0, masks=None, poison=True, spread=None):
    """A layer, cache planes whose unused rows are NaN, queries and masks; returns a dict."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    rng = np.random.default_rng(seed)
    B, n_h, r2 = len(lens), w.n_h, 2 * w.r
    kw = d_ck or w.d_c
    vw = w.d_c - d_ck if d_ck else w.d_c
    idx = gen.elite_index_sets(w)
    W_uk = (torch.randn((kw, n_h * w.d_nope), generator=g) * w.d ** -0.5).to(torch.bfloat16).cuda()
    W_uv = (torch.randn((vw, n_h * w.d_h), generator=g) * w.d ** -0.5).to(torch.bfloat16).cuda()
    layer = ek.Layer(n_h, w.d_h, w.r, w.d_c, idx, W_uk, W_uv, 64, d_ck=d_ck)
    fill = float("nan") if poison else 0.0
    if ps:
        need = [-(-n // ps) for n in lens]
        n_pages = spread or sum(need) + 3
        perm = rng.permutation(n_pages)[:sum(need)] if spread is None else n_pages - 1 - np.arange(sum(need))
        table = np.full((B, max(max(need), 1)), -1, dtype=np.int32)
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = perm[at:at + k]
            at += k
        where = [[int(table[b, t // ps]) * ps + t % ps for t in range(n)] for b, n in enumerate(lens)]
        rows, page_table, max_ctx = n_pages * ps, i32(table), 0
    else:
        max_ctx = max(max(lens), 1) + 3
        where = [[b * max_ctx + t for t in range(n)] for b, n in enumerate(lens)]
        rows, page_table = B * max_ctx, None
    rope = torch.full((rows, n_h * r2 or 8), fill, dtype=torch.bfloat16, device="cuda") if spread is None else \
        torch.zeros((rows, n_h * r2), dtype=torch.bfloat16, device="cuda")
    lat = torch.full((rows, w.d_c), fill, dtype=torch.bfloat16, device="cuda") if spread is None else \
        torch.zeros((rows, w.d_c), dtype=torch.bfloat16, device="cuda")
    flat = torch.tensor([x for v in where for x in v], dtype=torch.int64, device="cuda")
    k_vals = torch.randn((len(flat), n_h * r2), generator=g).to(torch.bfloat16).cuda()
    c_vals = torch.randn((len(flat), w.d_c), generator=g).to(torch.bfloat16).cuda()
    if r2:
        rope[flat] = k_vals
    lat[flat] = c_vals
    cache = ek.make_cache(rope, lat, n_seqs=B, max_ctx=max_ctx, page_table=page_table, page_size=ps or 64)
    std = scale_q * (w.d_nope / w.d) ** 0.5
    q_abs = (torch.randn((B, m, n_h, kw), generator=g) * std).to(torch.bfloat16).cuda()
    q_rope = (torch.randn((B, m, n_h, r2), generator=g) * scale_q).to(torch.bfloat16).cuda()
    if masks is None:
        parent = random_parents(rng, B, m)
        masks = np.array([T.mask_bits(parent[b], m) for b in range(B)], dtype=np.uint64)
    ws = torch.empty(ek.elitekv_attend_tree_workspace_size(layer, B, m), dtype=torch.uint8, device="cuda")
    return {"w": w, "layer": layer, "cache": cache, "rope": rope, "lat": lat, "q_abs": q_abs, "q_rope": q_rope, "lens": lens, "nodes": nodes,
            "mask": torch.from_numpy(np.asarray(masks, dtype=np.uint64).view(np.int64)).cuda(), "bits": masks, "W_uv": W_uv, "where": where,
            "kw": kw, "vw": vw, "ws": ws, "m": m, "page_table": page_table}


def call_tree(ek, s, **over):
    s = {**s, **over}
    out = ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32(s["lens"]),
                                 None if s["nodes"] is None else i32(s["nodes"]), s["mask"], s["ws"], s.get("out"))
    torch.cuda.synchronize()
    code = ek.elitekv_check_status(s["layer"])
    assert code == 0, ek.strerror(code)
    return out


def check_tree(s, out, heads=None, seqs=None, tol=TOL):
    w, m = s["w"], s["m"]
    heads = list(range(w.n_h)) if heads is None else heads
    num = den = 0.0
    for b in range(len(s["lens"])) if seqs is None else seqs:
        n, k = s["lens"][b], m if s["nodes"] is None else s["nodes"][b]
        got = H.f64(out[b])[:, heads]
        assert not got[k:].any()
        if n == 0 or k == 0:
            assert not got.any()
            continue
        at = torch.tensor(s["where"][b], device="cuda")
        kr = H.f64(s["rope"][at][:, :w.n_h * 2 * w.r]).reshape(n, w.n_h, 2 * w.r)[:, heads]
        c = H.f64(s["lat"][at])
        W = H.f64(s["W_uv"]).reshape(s["vw"], w.n_h, w.d_h)[:, heads].reshape(s["vw"], -1)
        want = T.attend_tree(H.f64(s["q_rope"][b, :k])[:, heads], H.f64(s["q_abs"][b, :k])[:, heads], kr, c[:, :s["kw"]], c[:, w.d_c - s["vw"]:],
                             W, n - k, s["bits"][b], w.d_h ** -0.5)
        fine = np.isfinite(want)
        assert np.array_equal(fine.all(-1), np.isfinite(got[:k]).all(-1)), b
        d = np.where(fine, got[:k] - np.where(fine, want, 0), 0)
        want = np.where(fine, want, 0)
        num += float((d ** 2).sum())
        den += float((want ** 2).sum())
        assert (np.abs(d) <= 4 * tol * np.abs(want).max(-1, keepdims=True) + 1e-30).all(), (b, np.abs(d).max())
    assert den == 0 or (num / den) ** 0.5 <= tol, (num / den) ** 0.5


ODD = replace(gen.TINY, n_h=5, d_h=24, r=3, d_c=40)
WIDE = replace(gen.LLAMA7B_75, n_h=6)
SHAPES = {
    "tiny": (gen.TINY, 0), "odd": (ODD, 0), "no-rope": (replace(gen.TINY, n_h=3, r=0, d_c=72), 0), "all-rope": (replace(gen.TINY, n_h=2, r=32), 0),
    "7b": (gen.LLAMA7B_75, 0), "13b": (gen.LLAMA13B_75, 0), "87.5": (gen.SWEEP_875, 0), "slrd": (gen.LLAMA7B_75, 512),
    "slrd-odd": (replace(gen.TINY, n_h=3, d_c=136), 40), "few-heads": (WIDE, 0), "one-head": (replace(gen.LLAMA7B_75, n_h=1, d_c=264), 0),
}


@pytest.mark.parametrize("ps", [0, 64, 16])
@pytest.mark.parametrize("m", [1, 2, 5, 16, 33, 64])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_tree_shapes(ek, shape, m, ps):
    """Every layer shape with every tree size: sequences without a prefix, of one token, of odd lengths on both sides of the
    64-, 128- and 256-token marks, ragged trees down to none, rows of the planes that belong to nobody full of NaN."""
    w, d_ck = SHAPES[shape]
    lens = [m, 300, 64 + m, 0, 255, 257, 129 + m, 1]
    nodes = [m, m, m // 2, 0, max(m - 1, 0), m, m, min(1, m)]
    s = tree_state(ek, w, lens, nodes, m, ps=ps, seed=m + ps, d_ck=d_ck)
    heads = None if w.n_h < 8 else [0, 1, w.n_h // 2, w.n_h - 1]
    check_tree(s, call_tree(ek, s), heads)


@pytest.mark.parametrize("ps", [1, 2, 4, 8, 32, 128, 512])
def test_tree_page_sizes(ek, ps):
    for w, d_ck in ((gen.TINY, 0), (gen.LLAMA7B_75, 0), (gen.LLAMA7B_75, 512)):
        s = tree_state(ek, w, [190, 7, 333], [7, 7, 3], 7, ps=ps, seed=ps, d_ck=d_ck)
        check_tree(s, call_tree(ek, s), [0, 3, w.n_h - 1])


@pytest.mark.parametrize("w", [gen.TINY, gen.LLAMA7B_75])
def test_tree_masks(ek, w):
    """Masks that no tree gives: a row that sees nothing of the tree, one that sees all of it, bits behind the last node, rows
    without a prefix that see nothing at all."""
    m = 6
    masks = np.array([[0, 63, 1 << 5, 1 << 63 | 2, 0b101, (1 << 64) - 1]] * 3, dtype=np.uint64)
    s = tree_state(ek, w, [200, 6, 4], [6, 6, 4], m, masks=masks, seed=5)
    out = call_tree(ek, s)
    check_tree(s, out, [0, 2])
    assert not out[1, 0].any() and out[0, 0].any()
    # no count given: m nodes everywhere
    s = tree_state(ek, w, [200, 6, 77], None, m, masks=masks, seed=6)
    check_tree(s, call_tree(ek, s), [0, 2])


@pytest.mark.parametrize("w,d_ck", [(gen.TINY, 0), (gen.LLAMA7B_75, 0), (gen.LLAMA7B_75, 512), (gen.SWEEP_875, 0)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(ek, w, d_ck, bad):
    m = 9
    parent = np.array([[-1, 0, 0, 1, 1, 2, 2, 5, 3]])
    masks = np.array([T.mask_bits(parent[0], m)], dtype=np.uint64)
    for n, node in ((140, 2), (m, 4), (64 + m, 8), (256 + 5, 1)):
        s = tree_state(ek, w, [n], [m], m, masks=masks, seed=n, d_ck=d_ck)
        at = s["where"][0][n - m + node]
        clean = call_tree(ek, s)
        s["lat"][at, w.d_c - 3] = bad
        if node % 2:
            s["rope"][at] = bad
        out = call_tree(ek, s)
        sees = [bool(int(masks[0, i]) >> node & 1) for i in range(m)]
        assert any(sees) and not all(sees)
        for i in range(m):
            if sees[i]:
                assert not torch.isfinite(out[0, i].float()).all(-1).any(), i
            else:
                assert torch.equal(out[0, i], clean[0, i]), i


@pytest.mark.parametrize("w", [gen.TINY, gen.LLAMA7B_75, gen.LLAMA13B_75])
@pytest.mark.parametrize("scale_q", [8.0, 64.0])
def test_peaked_scores(ek, w, scale_q):
    """Scores of up to hundreds of base-2 units, growing along the sequence: the reference of the softmax moves between and
    inside pieces, and one token dominates."""
    m = 3
    s = tree_state(ek, w, [1500, 700], [3, 2], m, seed=int(scale_q), scale_q=scale_q)
    for b in range(2):
        at = torch.tensor(s["where"][b], device="cuda")
        ramp = torch.linspace(0.1, 1.5, len(at), device="cuda")[:, None]
        s["lat"][at] = (s["lat"][at].float() * ramp).to(torch.bfloat16)
    check_tree(s, call_tree(ek, s), [0, 1, w.n_h - 1])
    # all scores far below zero, and one far above
    s["q_rope"].zero_()
    for b in range(2):
        at = torch.tensor(s["where"][b], device="cuda")
        u = s["q_abs"][b, 0, 0, :s["kw"]].float()
        s["lat"][at] = (s["lat"][at].float() * 0.1 - 4 * u / u.norm() * torch.linspace(1, 20, len(at), device="cuda")[:, None]).to(torch.bfloat16)
    check_tree(s, call_tree(ek, s), [0])
    s["lat"][s["where"][0][100]] *= -1
    s["lat"][s["where"][0][1300]] *= -1
    check_tree(s, call_tree(ek, s), [0])


def test_long_sequences(ek):
    """Several pieces and splits per sequence, every row tile size."""
    for w, m, lens, d_ck in ((gen.LLAMA7B_75, 4, [9001, 40, 5000], 0), (gen.LLAMA7B_75, 16, [4609, 2304], 0),
                             (gen.LLAMA13B_75, 7, [3000, 6000, 1], 0), (gen.LLAMA7B_75, 64, [2500], 512)):
        nodes = [min(m, n) for n in lens]
        s = tree_state(ek, w, lens, nodes, m, ps=64 if m == 16 else 0, seed=m, d_ck=d_ck)
        s["heads"] = [0, w.n_h - 1]
        check_tree(s, call_tree(ek, s), s["heads"])


def test_cache_rows_beyond_32_bit_offsets(ek):
    """Pages at the end of planes of more than 2^31 elements (bytes pass 2^32)."""
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [200, 90], [4, 2], 4, ps=64, seed=9, spread=23000)
    assert s["lat"].numel() > 2 ** 31
    check_tree(s, call_tree(ek, s), [0, 31])


def test_many_sequences(ek):
    w = gen.TINY
    rng = np.random.default_rng(0)
    lens = rng.integers(8, 90, 300).tolist()
    s = tree_state(ek, w, lens, rng.integers(0, 9, 300).tolist(), 8, ps=16, seed=1)
    check_tree(s, call_tree(ek, s), [0, 3], seqs=range(0, 300, 17))


def test_results_do_not_depend_on_scheduling_or_company(ek):
    """The same bits again, on another stream, with another kernel beside it, with garbage in workspace and output."""
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [3000, 1025, 64], [16, 9, 16], 16, seed=2)
    out = call_tree(ek, s).clone()
    x = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    for fill in (0, 255, 127):
        s["ws"].fill_(fill)
        s["out"] = torch.full_like(out, float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32(s["lens"]), i32(s["nodes"]), s["mask"],
                                         s["ws"], s["out"])
        y = x @ x
        torch.cuda.synchronize()
        assert torch.equal(got, out)
    del y
    assert ek.elitekv_check_status(s["layer"]) == 0


def test_two_calls_at_once(ek):
    """Two streams, two workspaces, both calls larger than the device."""
    w = gen.LLAMA7B_75
    a = tree_state(ek, w, [4000] * 4, [16] * 4, 16, seed=3)
    b = tree_state(ek, w, [3000] * 5, [12] * 5, 12, seed=4)
    want = [call_tree(ek, s).clone() for s in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    args = [(i32(s["lens"]), i32(s["nodes"]), torch.empty_like(w_)) for s, w_ in zip((a, b), want)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st, (lens, nodes, out) in zip((a, b), streams, args):
            with torch.cuda.stream(st):
                ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], lens, nodes, s["mask"], s["ws"], out)
    torch.cuda.synchronize()
    for s, (_, _, out), x in zip((a, b), args, want):
        assert ek.elitekv_check_status(s["layer"]) == 0
        assert torch.equal(out, x)


def test_lengths_and_pages_out_of_range_are_recorded(ek):
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [100, 50], [4, 4], 4, ps=64, seed=8)
    for lens, nodes, code in (([100, 5000], [4, 4], ek.ERR_BAD_POSITION), ([100, -3], [4, 4], ek.ERR_BAD_POSITION),
                              ([100, 50], [4, 5], ek.ERR_BAD_POSITION), ([100, 50], [-1, 4], ek.ERR_BAD_POSITION),
                              ([100, 2], [4, 3], ek.ERR_BAD_POSITION)):
        ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32(lens), i32(nodes), s["mask"], s["ws"])
        assert ek.elitekv_check_status(s["layer"]) == code, (lens, nodes)
    good = call_tree(ek, s).clone()
    s["page_table"][1, 0] = 1 << 20
    out = ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32([100, 50]), i32([4, 4]), s["mask"], s["ws"])
    assert ek.elitekv_check_status(s["layer"]) == ek.ERR_BAD_PAGE
    assert torch.equal(out[0], good[0])


def test_tree_refuses(ek):
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [100], [4], 4, seed=8)
    L, p, n = s["layer"], s["ws"].data_ptr(), s["ws"].numel()
    import ctypes as C
    q = s["q_abs"].data_ptr()
    lens, out = i32([100]), torch.empty((1, 4, 32, 128), dtype=torch.bfloat16, device="cuda")

    def call(layer=L.handle, cache=s["cache"], q_rope=s["q_rope"].data_ptr(), q_abs=q, lens_=lens.data_ptr(), mask=s["mask"].data_ptr(),
             B=1, m=4, ws=p, bytes_=n, out_=out.data_ptr()):
        return ek.lib().elitekv_attend_tree(layer, C.byref(cache) if cache else None, q_rope, q_abs, lens_, None, mask, B, m, ws, bytes_, out_, None)

    for bad in ({"q_rope": None}, {"q_abs": None}, {"lens_": None}, {"mask": None}, {"ws": None}, {"out_": None}, {"cache": None}, {"B": 0}, {"B": 2},
                {"m": 0}, {"m": 65}, {"q_abs": q + 2}, {"out_": out.data_ptr() + 2}, {"mask": s["mask"].data_ptr() + 4}):
        assert call(**bad) == ek.ERR_INVALID_ARG, bad
    assert call(bytes_=n - 1) == ek.ERR_WORKSPACE_TOO_SMALL and call(ws=p + 128) == ek.ERR_WORKSPACE_TOO_SMALL
    for m in (0, 65):
        with pytest.raises(ek.ElitekvError):
            ek.elitekv_attend_tree_workspace_size(L, 1, m)
    assert call() == 0
    torch.cuda.synchronize()


# ------------------------------------------------------------------------------- acceptance
@pytest.mark.parametrize("ps", [0, 16])
@pytest.mark.parametrize("B,m,w", [(1, 1, gen.TINY), (7, 16, gen.LLAMA7B_75), (40, 64, replace(gen.TINY, n_h=3, r=1)), (3, 33, replace(gen.TINY, r=0)),
                                   (2, 64, gen.LLAMA13B_75)])
def test_acceptance(ek, B, m, w, ps):
    rng = np.random.default_rng(B * 100 + m)
    held = rng.integers(0, 50, B).tolist()
    nodes = rng.integers(0, m + 1, B).tolist()
    nodes[0] = m
    s = tree_state(ek, w, [h + m for h in held], [m] * B, m, ps=ps, seed=B + m, poison=False)
    parent = random_parents(rng, B, m)
    if B == 2:
        parent[1] = np.arange(m) - 1
    draft = rng.integers(0, 4, (B, m))                     # few tokens: siblings that draft the same
    chosen = rng.integers(0, 4, (B, m))
    for b in range(B):
        for i in range(m):
            if rng.random() < 0.7 or B == 2:
                chosen[b, max(int(parent[b, i]), 0)] = draft[b, i]
    first = draft[:, 0].copy()
    first[B // 2] = draft[B // 2, 0] if B < 3 else 9       # nothing accepted
    rope, lat = s["rope"].clone(), s["lat"].clone()
    got = ek.elitekv_accept_tree(s["layer"], s["cache"], i32(held), i32(nodes), i32(parent), i32(draft), i32(first), i32(chosen))
    assert ek.elitekv_check_status(s["layer"]) == 0
    longest = 0
    for b in range(B):
        path, want = T.accept(parent[b], draft[b], first[b], chosen[b], nodes[b])
        longest = max(longest, len(path))
        assert got[0][b] == len(path) and got[1][b].tolist() == path + [-1] * (m - len(path))
        assert got[2][b] == want and got[3][b] == held[b] + len(path)
        for plane, was in ((s["rope"], rope), (s["lat"], lat)):
            for k, i in enumerate(path):
                assert torch.equal(plane[s["where"][b][held[b] + k]], was[s["where"][b][held[b] + i]])
            keep = [x for t, x in enumerate(s["where"][b]) if t < held[b] or t >= held[b] + len(path)]
            assert torch.equal(plane[keep], was[keep])
    assert longest > 1 or m == 1


def test_acceptance_in_place_and_as_a_chain(ek):
    w, m = gen.TINY, 5
    s = tree_state(ek, w, [20, 20], [m, m], m, poison=False)
    held, first = i32([10, 12]), i32([1, 4])
    draft, chosen = i32([[1, 2, 3, 4, 5], [1, 2, 3, 4, 5]]), i32([[2, 3, 9, 5, 6], [2, 3, 4, 5, 6]])
    before = s["lat"].clone()
    n, path, token, out = ek.elitekv_accept_tree(s["layer"], s["cache"], held, None, None, draft, first, chosen, token=first, held_out=held)
    assert n.tolist() == [3, 0] and token.tolist() == [9, 4] and held.tolist() == [13, 12] and out is held
    assert torch.equal(s["lat"], before)                   # a chain's rows are in place


def test_acceptance_records_bad_pages(ek):
    w, m = gen.TINY, 4
    s = tree_state(ek, w, [40], [m], m, ps=16, poison=False)
    s["page_table"][0, 2] = 999
    parent, draft, chosen = i32([[-1, 0, 0, 2]]), i32([[1, 2, 3, 4]]), i32([[3, 0, 4, 7]])
    n, path, token, out = ek.elitekv_accept_tree(s["layer"], s["cache"], i32([36]), None, parent, draft, i32([1]), chosen)
    assert ek.elitekv_check_status(s["layer"]) == ek.ERR_BAD_PAGE
    assert path.tolist() == [[0, 2, 3, -1]] and out.tolist() == [39]
    # lengths past the cache
    ek.elitekv_accept_tree(s["layer"], s["cache"], i32([47]), None, parent, draft, i32([1]), chosen)
    assert ek.elitekv_check_status(s["layer"]) != 0


# ------------------------------------------------------------------------------- in a row
class Loop:
    """What a serving loop keeps for its speculative steps: device buffers only, so that a step can be captured."""

    def __init__(self, ek, w, B, m, held, ps, seed, d_ck=0):
        self.ek, self.w, self.B, self.m = ek, w, B, m
        g = torch.Generator(device="cpu").manual_seed(seed)
        kw, vw = (d_ck, w.d_c - d_ck) if d_ck else (w.d_c, w.d_c)
        self.idx, self.d_ck = gen.elite_index_sets(w), d_ck
        self.W_uk = (torch.randn((kw, w.n_h * w.d_nope), generator=g) * w.d ** -0.5).to(torch.bfloat16).cuda()
        self.W_uv = (torch.randn((vw, w.n_h * w.d_h), generator=g) * w.d ** -0.5).to(torch.bfloat16).cuda()
        self.layer = ek.Layer(w.n_h, w.d_h, w.r, w.d_c, self.idx, self.W_uk, self.W_uv, 4096, d_ck=d_ck)
        pages = [-(-h // ps) for h in held]
        n_pages = sum(pages) + 40
        perm = np.random.default_rng(seed).permutation(n_pages)
        table = np.full((B, max(pages) + 8), -1, dtype=np.int32)
        at = 0
        for b, k in enumerate(pages):
            table[b, :k] = perm[at:at + k]
            at += k
        self.table, self.ps = i32(table), ps
        self.rope = torch.full((n_pages * ps, w.n_h * 2 * w.r), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.lat = torch.full((n_pages * ps, w.d_c), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.cache = ek.make_cache(self.rope, self.lat, n_seqs=B, page_table=self.table, page_size=ps)
        self.held, self.fresh, self.first = i32(held), i32([m] * B), i32([0] * B)
        self.pages, self.free, self.n_free = i32(pages), i32(perm[at:]), i32([n_pages - at])
        self.parent = i32(np.zeros((B, m)))
        self.draft, self.chosen = i32(np.zeros((B, m))), i32(np.zeros((B, m)))
        self.k_e = torch.zeros((B * m, w.n_h, w.r, 2), dtype=torch.bfloat16, device="cuda")
        self.c = torch.zeros((B * m, w.d_c), dtype=torch.bfloat16, device="cuda")
        self.q = torch.zeros((B * m, w.n_h, w.d_h), dtype=torch.bfloat16, device="cuda")
        self.q_rope = torch.zeros((B * m, w.n_h, 2 * w.r), dtype=torch.bfloat16, device="cuda")
        self.q_abs = torch.zeros((B * m, w.n_h, kw), dtype=torch.bfloat16, device="cuda")
        self.t = ek.make_tables(B, B * m, m, self.held, self.fresh, parent=self.parent, page_table=self.table, pages_held=self.pages,
                                free_pages=self.free, n_free=self.n_free)
        self.ws = torch.empty(ek.elitekv_attend_tree_workspace_size(self.layer, B, m), dtype=torch.uint8, device="cuda")
        self.out = torch.zeros((B, m, w.n_h, w.d_h), dtype=torch.bfloat16, device="cuda")
        self.n_acc, self.path = i32([0] * B), i32(np.zeros((B, m)))

    def prompt(self, tokens):
        """The committed tokens (k_e, c per sequence) through a packed step."""
        held = self.held.tolist()
        zero = i32([0] * self.B)
        t = self.ek.make_tables(self.B, sum(held) + 2, 0, zero, self.held, page_table=self.table, pages_held=self.pages,
                                free_pages=self.free, n_free=self.n_free)
        self.ek.elitekv_step_tables(self.cache, t)
        assert t.result.tolist() == [0, sum(held), 0, 0]
        pad = [torch.zeros_like(x[:2]) for x in tokens]
        self.ek.elitekv_append_slots(self.layer, self.cache, torch.cat([tokens[0], pad[0]]), torch.cat([tokens[1], pad[1]]), t.slot, t.pos)

    def step(self):
        ek, B, m, w = self.ek, self.B, self.m, self.w
        ek.elitekv_step_tables(self.cache, self.t)
        ek.elitekv_append_slots(self.layer, self.cache, self.k_e, self.c, self.t.slot, self.t.pos)
        ek.elitekv_absorb_query(self.layer, self.q, self.t.pos, self.q_rope, self.q_abs)
        ek.elitekv_attend_tree(self.layer, self.cache, self.q_rope.view(B, m, w.n_h, -1), self.q_abs.view(B, m, w.n_h, -1), self.t.seq_lens,
                               self.fresh, self.t.tree_mask, self.ws, self.out)
        ek.elitekv_accept_tree(self.layer, self.cache, self.held, self.fresh, self.parent, self.draft, self.first, self.chosen,
                               self.n_acc, self.path, self.first, self.held)
        self.pages.copy_(self.t.pages_held_out)
        self.n_free.copy_(self.t.n_free_out)


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("w,d_ck", [(gen.TINY, 0), (gen.LLAMA7B_75, 0), (gen.LLAMA7B_75, 512)])
def test_speculative_steps_in_a_row(ek, w, d_ck, graph):
    """Five steps over a paged cache, captured once and replayed: every node's attention is what the oracle says of its own
    branch (raw keys rotated at their depth), and after each step the cache decodes like one that held the accepted
    tokens all along."""
    B, m, ps = 3, 7, 16
    held = [21, 5, 48]
    lp = Loop(ek, w, B, m, held, ps, seed=3, d_ck=d_ck)
    g = torch.Generator(device="cpu").manual_seed(77)
    rng = np.random.default_rng(7)
    hist_k = [torch.randn((h, w.n_h, w.r, 2), generator=g).to(torch.bfloat16) for h in held]
    hist_c = [torch.randn((h, w.d_c), generator=g).to(torch.bfloat16) for h in held]
    lp.prompt((torch.cat(hist_k).cuda(), torch.cat(hist_c).cuda()))
    want_first = [0] * B
    cg = None
    idx = lp.idx.numpy().astype(np.int64)
    W_uk, W_uv = H.f64(lp.W_uk), H.f64(lp.W_uv)
    dq = w.d_c - (w.d_c - d_ck if d_ck else w.d_c)

    def attend(q, pos, k, c, heads):
        k, c = H.f64(k), H.f64(c)
        kr = O.rotate_elite_keys(k, np.arange(len(k)), idx, w.d_h)
        if d_ck:
            return O.decode_slrd(H.f64(q), pos, kr, c[:, :d_ck], c[:, dq:], W_uk, W_uv, idx, w.d_h, heads=heads)
        return O.decode(H.f64(q), pos, kr, c, W_uk, W_uv, idx, w.d_h, heads=heads)

    heads = [0, w.n_h - 1]
    for it in range(5):
        parent = random_parents(rng, B, m)
        parent[:, 0] = -1
        fresh = rng.integers(1, m + 1, B)
        draft, chosen = rng.integers(0, 3, (B, m)), rng.integers(0, 3, (B, m))
        for b in range(B):
            draft[b, 0] = want_first[b]
            for i in range(1, m):
                if rng.random() < 0.7:
                    chosen[b, max(int(parent[b, i]), 0)] = draft[b, i]
        k_e = torch.randn((B, m, w.n_h, w.r, 2), generator=g).to(torch.bfloat16)
        c = torch.randn((B, m, w.d_c), generator=g).to(torch.bfloat16)
        q = torch.randn((B, m, w.n_h, w.d_h), generator=g).to(torch.bfloat16)
        if graph and it == 1:
            torch.cuda.synchronize()
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                lp.step()
        lp.fresh.copy_(i32(fresh))
        lp.parent.copy_(i32(parent))
        lp.draft.copy_(i32(draft))
        lp.chosen.copy_(i32(chosen))
        lp.k_e.copy_(k_e.view_as(lp.k_e))
        lp.c.copy_(c.view_as(lp.c))
        lp.q.copy_(q.view_as(lp.q))
        cg.replay() if cg is not None else lp.step()
        torch.cuda.synchronize()
        assert ek.elitekv_check_status(lp.layer) == 0 and lp.t.result[0] == 0
        for b in range(B):
            num = den = 0.0
            for i in range(int(fresh[b])):
                line = sorted(T.ancestors(parent[b], i))
                want = attend(q[b, i], len(hist_k[b]) + len(line) - 1, torch.cat([hist_k[b], k_e[b, line]]), torch.cat([hist_c[b], c[b, line]]), heads)
                got = H.f64(lp.out[b, i])[heads]
                num, den = num + ((got - want) ** 2).sum(), den + (want ** 2).sum()
            assert (num / den) ** 0.5 <= H.REL_L2_TOL, (it, b, (num / den) ** 0.5)     # bf16 rows and queries in between
            path, want_first[b] = T.accept(parent[b], draft[b], want_first[b], chosen[b], int(fresh[b]))
            assert lp.path[b].tolist()[:len(path)] == path and int(lp.n_acc[b]) == len(path)
            hist_k[b] = torch.cat([hist_k[b], k_e[b, path]])
            hist_c[b] = torch.cat([hist_c[b], c[b, path]])
        assert lp.held.tolist() == [len(x) for x in hist_k] and lp.first.tolist() == want_first
    # a decode step of the library over the cache that the trees left
    q1 = torch.randn((B, w.n_h, w.d_h), generator=g).to(torch.bfloat16)
    q_rope, q_abs = ek.elitekv_absorb_query(lp.layer, q1.cuda(), lp.held - 1)
    dws = torch.empty(ek.elitekv_decode_workspace_size(lp.layer, B), dtype=torch.uint8, device="cuda")
    out = ek.elitekv_decode(lp.layer, lp.cache, q_rope, q_abs, lp.held, dws)
    assert ek.elitekv_check_status(lp.layer) == 0
    for b in range(B):
        want = attend(q1[b], len(hist_k[b]) - 1, hist_k[b], hist_c[b], heads)
        rel, mx = H.errors(H.f64(out[b])[heads], want)
        assert rel <= H.REL_L2_TOL and mx <= H.MAX_ABS_TOL, (b, rel, mx)


def test_chain_is_the_query_rows_call(ek):
    """A chain gives what elitekv_attend_rows gives, to the roundings of both."""
    w, m = gen.LLAMA7B_75, 4
    s = tree_state(ek, w, [500, 131], None, m, masks=np.array([T.mask_bits(None, m)] * 2, dtype=np.uint64), seed=12)
    out = call_tree(ek, s)
    ws = torch.empty(ek.elitekv_attend_rows_workspace_size(s["layer"], 2, m), dtype=torch.uint8, device="cuda")
    rows = ek.elitekv_attend_rows(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32(s["lens"]), m, ws)
    torch.cuda.synchronize()
    rel, _ = H.errors(H.f64(out), H.f64(rows))
    assert rel <= 2 * TOL
