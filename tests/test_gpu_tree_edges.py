"""GPU parity of tree attention where its kernels change hands or cut their work: one node, the smallest calls, many runs
and chained pieces, head dims at both ends, captured calls that share a workspace.  Tolerances are those of
tests/test_gpu_tree.py (two bf16 roundings), against the same float64 oracle."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import tree_oracle as T
from paper_2503_01586_b200 import inputs as gen

from .test_gpu_tree import ODD, call_tree, check_tree, ek, i32, tree_state  # noqa: F401  (ek is a fixture)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------- one node
@pytest.mark.parametrize("w,d_ck", [(gen.TINY, 0), (ODD, 0), (gen.LLAMA7B_75, 0), (gen.LLAMA7B_75, 512), (gen.SWEEP_875, 0)])
@pytest.mark.parametrize("ps", [0, 1, 16, 64])
def test_one_node(ek, w, d_ck, ps):
    """A node that does not see itself, one that sees itself only, one that sees nothing, none at all, and bits behind it."""
    lens, nodes = [70, 70, 1, 1, 33, 0, 300], [1, 1, 1, 1, 0, 0, 1]
    masks = np.array([[0], [1], [1], [0], [1], [1], [(1 << 64) - 1]], dtype=np.uint64)
    s = tree_state(ek, w, lens, nodes, 1, ps=ps, masks=masks, seed=ps, d_ck=d_ck)
    heads = [0, w.n_h - 1]
    out = call_tree(ek, s)
    check_tree(s, out, heads)
    assert not out[[3, 4, 5]].any() and out[[0, 1, 2, 6]].any(-1).all()
    # what a node does not see may be anything
    at = s["where"][0][69]
    s["lat"][at] = float("nan")
    s["rope"][at] = float("inf")
    again = call_tree(ek, s)
    assert torch.equal(again, out)
    # all lengths a sequence may have, and none beyond
    if ps == 0:
        s["nodes"] = None
        for bad in (-1, s["cache"].max_ctx + 1):
            ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32([70, bad] + lens[2:]), None, s["mask"], s["ws"])
            assert ek.elitekv_check_status(s["layer"]) == ek.ERR_BAD_POSITION


# ------------------------------------------------------------------------------- sizes at which another kernel takes over
@pytest.mark.parametrize("w,m,n", [(gen.TINY, 7, 637), (gen.TINY, 7, 638), (gen.TINY, 64, 197), (gen.TINY, 64, 198), (gen.LLAMA7B_75, 2, 253),
                                   (gen.LLAMA7B_75, 2, 254), (gen.SWEEP_875, 4, 225), (gen.SWEEP_875, 4, 226), (gen.LLAMA7B_75, 64, 70)])
def test_small_calls(ek, w, m, n):
    """Capacities (three tokens more than the longest sequence) just within and just past what the kernel for small calls
    takes, with a tree whose masks hide most of it."""
    rng = np.random.default_rng(n)
    parent = np.where(rng.random((1, m)) < 0.5, -1, np.maximum(np.arange(m) - 1 - rng.integers(0, 3, m), -1))
    masks = np.array([T.mask_bits(parent[0], m)], dtype=np.uint64)
    s = tree_state(ek, w, [n], [m], m, masks=masks, seed=n)
    check_tree(s, call_tree(ek, s), [0, w.n_h - 1])


def test_tokens_in_flight_around_a_branch(ek):
    """Every phase of the prefix against the groups of tokens that a warp takes at once, drafted rows of others not finite."""
    w, m = gen.TINY, 5
    masks = np.array([[0b00001, 0b00010, 0b10101, 0, 0b11111]], dtype=np.uint64)
    for n in range(m, m + 10):
        s = tree_state(ek, w, [n], [m], m, masks=masks, seed=n)
        clean = call_tree(ek, s)
        check_tree(s, clean)
        s["lat"][s["where"][0][n - 4]] = float("nan")          # node 1
        out = call_tree(ek, s)
        assert torch.equal(out[0, [0, 2, 3]], clean[0, [0, 2, 3]]) and out[0, [1, 4]].isnan().all()


# ------------------------------------------------------------------------------- runs and pieces
@pytest.mark.parametrize("w,m,lens,d_ck", [(gen.LLAMA7B_75, 4, [40001], 0), (gen.LLAMA7B_75, 16, [30000, 300], 0), (gen.TINY, 33, [70001, 5], 0),
                                           (gen.LLAMA7B_75, 33, [20011], 512), (gen.SWEEP_875, 2, [33000, 16001], 0)])
@pytest.mark.parametrize("scale_q", [1.0, 40.0])
def test_many_runs_and_pieces(ek, w, m, lens, d_ck, scale_q):
    """More runs than a row keeps weights of, runs of several pieces; with large queries and growing latents the softmax
    reference moves from piece to piece."""
    nodes = [m, min(m, 5)][:len(lens)]
    s = tree_state(ek, w, lens, nodes, m, ps=0 if m == 4 else 64, seed=m, d_ck=d_ck, scale_q=scale_q)
    if scale_q > 1:
        for b in range(len(lens)):
            at = torch.tensor(s["where"][b], device="cuda")
            for i in range(0, len(at), 8192):
                ramp = torch.linspace(0.1 + 1.4 * i / len(at), 0.1 + 1.4 * min(1, (i + 8192) / len(at)), len(at[i:i + 8192]), device="cuda")[:, None]
                s["lat"][at[i:i + 8192]] = (s["lat"][at[i:i + 8192]].float() * ramp).to(torch.bfloat16)
    check_tree(s, call_tree(ek, s), [1])


# ------------------------------------------------------------------------------- shapes of the last product
def layer_of(n_h, d_h, r, d_c):
    return replace(gen.TINY, n_h=n_h, d_h=d_h, r=r, d_c=d_c, d=n_h * d_h)


@pytest.mark.parametrize("n_h,d_h,r,d_c,d_ck", [(4, 16, 1, 64, 0), (8, 16, 4, 328, 0), (4, 256, 8, 200, 0), (2, 256, 2, 640, 0), (12, 96, 3, 384, 0),
                                                (4, 48, 5, 392, 8), (4, 80, 2, 1032, 520), (16, 64, 4, 8, 0), (40, 32, 1, 136, 0), (3, 112, 4, 904, 0),
                                                (2, 512, 2, 72, 0)])
@pytest.mark.parametrize("m", [3, 40, 41, 43])
def test_head_dims_and_latents(ek, n_h, d_h, r, d_c, d_ck, m):
    """Head dims from 16 to 256, latents that end inside a tile of 64, 128 and 256 columns, tree sizes that leave 128-row
    blocks with 2 to 8 rows over."""
    w = layer_of(n_h, d_h, r, d_c)
    lens, nodes = [700, 43, 1300, 512], [m, m, max(m - 2, 1), m]
    s = tree_state(ek, w, lens, nodes, m, ps=32 if m & 1 else 0, seed=m + n_h, d_ck=d_ck)
    check_tree(s, call_tree(ek, s), [0, n_h - 1])


# ------------------------------------------------------------------------------- calls as programs make them
@pytest.mark.parametrize("m", [1, 3, 16])
def test_no_sequence_has_a_node(ek, m):
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [900, 0, 800], [0, 0, 0], m, seed=1)
    s["out"] = torch.full((3, m, w.n_h, w.d_h), float("nan"), dtype=torch.bfloat16, device="cuda")
    assert not call_tree(ek, s).any()


@pytest.mark.parametrize("m", [1, 2, 12])
def test_sequences_that_share_pages(ek, m):
    """A common prompt in the same pages of two sequences, and a cache that holds more sequences than the call."""
    w, ps = gen.LLAMA7B_75, 16
    s = tree_state(ek, w, [320 + 30, 320 + 17, 40], [m] * 3, m, ps=ps, seed=m)
    s["page_table"][1, :20] = s["page_table"][0, :20]
    s["where"][1][:320] = s["where"][0][:320]
    s["cache"].n_seqs = 3
    check_tree(s, call_tree(ek, s), [0, 31])
    two = {**s, "lens": s["lens"][:2], "nodes": s["nodes"][:2], "mask": s["mask"][:2].contiguous(), "q_abs": s["q_abs"][:2].contiguous(),
           "q_rope": s["q_rope"][:2].contiguous()}
    check_tree(two, call_tree(ek, two), [0, 31])


def test_captured_calls_that_share_a_workspace(ek):
    """Graphs of calls of different sizes over one workspace, replayed in turn on one stream, with lengths, nodes and masks
    that change between replays."""
    w = gen.LLAMA7B_75
    cases = [tree_state(ek, w, lens, nodes, m, ps=16, seed=20 + m) for lens, nodes, m in
             (([1500, 900], [16, 9], 16), ([77, 200, 5000], [3, 2, 3], 3), ([64, 130], [1, 1], 1), ([3000], [40], 40), ([90], [2], 2))]
    ws = torch.empty(max(s["ws"].numel() for s in cases), dtype=torch.uint8, device="cuda")
    graphs, state = [], []
    for s in cases:
        want = call_tree(ek, s).clone()
        lens, nodes, out = i32(s["lens"]), i32(s["nodes"]), torch.zeros_like(want)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], lens, nodes, s["mask"], ws, out)
        graphs.append(g)
        state.append((lens, nodes, out, want))
    for turn in range(3):
        ws.fill_((0, 255, 91)[turn])
        for g in graphs:
            g.replay()
        for g in reversed(graphs):
            g.replay()
        torch.cuda.synchronize()
        for s, (lens, nodes, out, want) in zip(cases, state):
            assert ek.elitekv_check_status(s["layer"]) == 0
            assert torch.equal(out, want)
            out.zero_()
    for s, g, (lens, nodes, out, _) in zip(cases, graphs, state):
        shorter = [max(n // 3, k) for n, k in zip(s["lens"], s["nodes"])]
        lens.copy_(i32(shorter))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        want = call_tree(ek, s, lens=shorter)
        assert torch.equal(out, want)


def test_calls_in_a_row_without_a_pause(ek):
    """Twenty calls of two sizes after one another on one stream and workspace: each starts while the last one ends."""
    w = gen.LLAMA7B_75
    a = tree_state(ek, w, [2500, 40], [5, 5], 5, seed=31)
    b = tree_state(ek, w, [300] * 9, [17] * 9, 17, seed=32)
    want = [call_tree(ek, s).clone() for s in (a, b)]
    ws = torch.empty(max(a["ws"].numel(), b["ws"].numel()), dtype=torch.uint8, device="cuda")
    args = [(i32(s["lens"]), i32(s["nodes"])) for s in (a, b)]
    outs = []
    for _ in range(10):
        for s, (lens, nodes) in zip((a, b), args):
            outs.append(ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], lens, nodes, s["mask"], ws))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert torch.equal(o, want[i % 2])


# ------------------------------------------------------------------------------- the other three, as programs make them
def test_tables_and_acceptance_on_another_stream_and_captured(ek):
    """The two calls before and after the attention, captured on a side stream beside a busy device: the same integers each
    time, and rows behind the accepted ones as they were."""
    w, B, m, ps = gen.TINY, 3, 6, 8
    s = tree_state(ek, w, [30 + m, 9 + m, m], [m] * B, m, ps=ps, seed=40, poison=False)
    held, fresh = i32([30, 9, 0]), i32([m, 4, 0])
    need = [-(-(h + m) // ps) for h in (30, 9, 0)]
    parent = i32([[-1, 0, 0, 1, 2, 2]] * B)
    draft, first, chosen = i32([[1, 2, 3, 4, 5, 6]] * B), i32([1, 1, 1]), i32([[3, 0, 6, 0, 0, 7]] * B)
    t = ek.make_tables(B, B * m, m, held, fresh, parent=parent, page_table=s["page_table"], pages_held=i32(need), free_pages=i32([0]),
                       n_free=i32([0]))
    lat = s["lat"].clone()
    res = [torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, m), dtype=torch.int32, device="cuda"),
           torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")]

    def step():
        ek.elitekv_step_tables(s["cache"], t)
        ek.elitekv_accept_tree(s["layer"], s["cache"], held, fresh, parent, draft, first, chosen, *res)

    step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    x = torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        s["lat"].copy_(lat)
        for y in res:
            y.fill_(-5)
        torch.cuda.synchronize()
        y = x @ x
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        assert ek.elitekv_check_status(s["layer"]) == 0 and t.result[0] == 0 and t.seq_lens.tolist() == [36, 13, 0]
        assert res[0].tolist() == [3, 2, 0] and res[3].tolist() == [33, 11, 0]
        assert res[1].tolist() == [[0, 2, 5, -1, -1, -1], [0, 2, -1, -1, -1, -1], [-1] * 6] and res[2].tolist() == [7, 6, 1]
        for b, path in ((0, [0, 2, 5]), (1, [0, 2]), (2, [])):
            h = (30, 9, 0)[b]
            for k, i in enumerate(path):
                assert torch.equal(s["lat"][s["where"][b][h + k]], lat[s["where"][b][h + i]])
            keep = [x_ for t_, x_ in enumerate(s["where"][b]) if not h <= t_ < h + len(path)]
            assert torch.equal(s["lat"][keep], lat[keep])
    del y


# ------------------------------------------------------------------------------- nodes as query rows of the decode kernel
@pytest.mark.parametrize("ps", [0, 64])
@pytest.mark.parametrize("w,d_ck", [(gen.LLAMA7B_75, 0), (gen.LLAMA13B_75, 0), (gen.LLAMA7B_75, 512), (gen.SWEEP_875, 0), (layer_of(8, 64, 4, 128), 0),
                                    (layer_of(24, 64, 16, 256), 128)])
@pytest.mark.parametrize("m", [2, 7, 15, 16])
def test_few_nodes_and_tokens(ek, w, d_ck, m, ps):
    """Trees across the marks of 16 and 128 tokens, with masks that hide any of their nodes, and hidden or padding rows that are
    not finite."""
    rng = np.random.default_rng(m + ps)
    for n in (m, 128, 128 + m // 2, 112 + m, 513):
        masks = (rng.integers(0, 1 << m, (2, m)) & ~1).astype(np.uint64)       # nobody sees node 0
        masks[0, m - 1] = 0
        s = tree_state(ek, w, [n, n - 1], [m, m - 1], m, ps=ps, masks=masks, seed=n, d_ck=d_ck)
        for b in range(2):
            s["lat"][s["where"][b][s["lens"][b] - s["nodes"][b]]] = float("nan")
        check_tree(s, call_tree(ek, s), [0, w.n_h - 1])
        if n > m:                                                               # what all nodes see, but for the padding one
            s["rope"][s["where"][1][0]] = s["lat"][s["where"][1][0]] = float("inf")
            out = call_tree(ek, s)
            assert not out[1, m - 1].any() and not torch.isfinite(out[1, :m - 1].float()).all(-1).any()


@pytest.mark.parametrize("m", [2, 5, 16])
def test_bad_lengths_of_few_nodes(ek, m):
    """The same records and rows as in longer calls."""
    w = gen.LLAMA7B_75
    s = tree_state(ek, w, [200, 50], [m, m], m, seed=8)
    good = call_tree(ek, s).clone()
    for lens, nodes in (([200, 5000], [m, m]), ([200, -3], [m, m]), ([200, 50], [m, m + 1]), ([200, 50], [m, -1]), ([200, 1], [m, m]), ([200, 0], [m, m])):
        out = ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], i32(lens), i32(nodes), s["mask"], s["ws"])
        assert ek.elitekv_check_status(s["layer"]) == ek.ERR_BAD_POSITION, (lens, nodes)
        assert ek.elitekv_last_status_detail(s["layer"])[0] == 1
        assert torch.equal(out[0], good[0])
        if lens[1] <= 0 or nodes[1] < 0:
            assert not out[1].any()


# ------------------------------------------------------------------------------- trees of one call that differ in size
@pytest.mark.parametrize("w,d_ck,m", [(gen.LLAMA7B_75, 0, 64), (gen.LLAMA7B_75, 0, 21), (gen.LLAMA7B_75, 512, 64), (gen.LLAMA13B_75, 0, 33),
                                      (gen.SWEEP_875, 0, 50), (layer_of(12, 64, 4, 200), 0, 64), (layer_of(80, 32, 2, 64), 0, 64),
                                      (layer_of(20, 48, 0, 72), 0, 64), (layer_of(6, 256, 2, 136), 8, 64)])
def test_ragged_trees(ek, w, d_ck, m):
    """Every number of nodes from none to m in one call, in runs of several pieces and in short ones; the rows behind a
    sequence's nodes are zero, whatever their queries hold, and a sequence's result is that of a call of its own."""
    rng = np.random.default_rng(m)
    nodes = [m, 0] + sorted(rng.permutation(np.arange(1, m))[:14].tolist()) + [1, m // 2, m // 2 + 1, m // 4, m - 1]
    lens = [int(k + rng.integers(0, 700)) if k % 3 else k + (2600 if k in (m, 1) else 0) for k in nodes]
    s = tree_state(ek, w, lens, nodes, m, ps=32, seed=m, d_ck=d_ck)
    for b, k in enumerate(nodes):
        s["q_abs"][b, k:] = float("nan")
        s["q_rope"][b, k:] = float("inf")
    out = call_tree(ek, s)
    check_tree(s, out, [0, w.n_h - 1])
    again = call_tree(ek, s)
    assert torch.equal(out, again)


def test_tables_of_lengths_that_pass_31_bits(ek):
    """A page table wide enough for 2^32 tokens, a sequence whose new length is no int32: refused before its pages are read."""
    table = i32(np.full((1, 8), -1))
    plane = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    cache = ek.make_cache(plane, plane, n_seqs=1, page_table=table, page_size=128)
    cache.max_pages_per_seq, cache.num_pages = 1 << 25, 1 << 25
    t = ek.make_tables(1, 16, 0, i32([(1 << 31) - 3]), i32([5]), page_table=table, pages_held=i32([1 << 24]), free_pages=i32([0]), n_free=i32([0]))
    ek.elitekv_step_tables(cache, t)
    assert t.result.tolist() == [ek.ERR_BAD_POSITION, 0, 0, 0] and t.slot.tolist() == [-1] * 16 and t.seq_lens.tolist() == [(1 << 31) - 3]


@pytest.mark.parametrize("w,d_ck", [(gen.LLAMA7B_75, 0), (gen.LLAMA13B_75, 0), (gen.LLAMA7B_75, 512), (gen.TINY, 0)])
@pytest.mark.parametrize("ps", [4, 8, 32])
def test_one_node_over_small_pages(ek, w, d_ck, ps):
    """Pages that no decode kernel on the tensor cores takes."""
    s = tree_state(ek, w, [3000, 1, 700], [1, 1, 0], 1, ps=ps, masks=np.array([[1], [1], [1]], dtype=np.uint64), seed=ps, d_ck=d_ck)
    check_tree(s, call_tree(ek, s), [0, w.n_h - 1])
