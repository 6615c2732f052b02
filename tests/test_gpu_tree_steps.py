"""Step tables that are refused, and what the calls behind them make of it."""
import numpy as np
import pytest
import torch

from oracle import tree_oracle as T
from paper_2503_01586_b200 import inputs as gen

from .test_gpu_tree import Loop, check_tables, ek, i32, run_tables  # noqa: F401  (ek is a fixture)

pytestmark = pytest.mark.gpu

LARGEST = 2 ** 31 - 1


# ------------------------------------------------------------------------------- page ids
@pytest.mark.parametrize("m", [0, 4])
@pytest.mark.parametrize("where", ["free", "table", "both"])
def test_the_largest_int_is_no_page(ek, m, where):
    """The largest int32, a common mark of "no page", among the pages that new tokens go to: refused as any id outside the
    pool.  With another bad id beside it the smaller one is named."""
    held, fresh = [3, 8], [4, 3]
    table, free = np.array([[2, -1, -1], [5, 1, -1]], dtype=np.int32), [7, 6, 4]
    if where != "table":
        free[1] = LARGEST
    if where != "free":
        table[0, 0] = 9 if where == "both" else LARGEST
    t, dev = run_tables(ek, held, fresh, m=m, n_slots=8, table=table, ps=4, pages_held=[1, 2], free=free, n_pages=8)
    assert t.result.tolist() == [ek.ERR_BAD_PAGE, 0, 0, 9 if where == "both" else LARGEST]
    assert np.array_equal(dev.cpu().numpy(), table) and t.slot.tolist() == [-1] * 8
    assert t.pages_held_out.tolist() == [1, 2] and t.n_free_out.tolist() == [3] and t.seq_lens.tolist() == held


def test_the_largest_int_where_no_new_token_goes(ek):
    """Below the pages that the step takes, and in a page whose tokens were there before."""
    held, fresh, table, free = [8, 8], [1, 3], np.array([[LARGEST, 3, -1], [5, 1, -1]], dtype=np.int32), [LARGEST, 6, 4]
    t, dev = run_tables(ek, held, fresh, m=0, n_slots=4, table=table, ps=4, pages_held=[2, 2], free=free, n_pages=8)
    check_tables(t, dev, T.step_tables(held, fresh, m=0, n_slots=4, page_table=table, page_size=4, pages_held=[2, 2], free_pages=free))


# ------------------------------------------------------------------------------- what a step was granted
@pytest.mark.parametrize("m", [0, 4])
def test_granted(ek, m):
    held, fresh, table = [3, 8, 0], [4, 3, 0], np.array([[2, -1, -1], [5, 1, -1], [-1, -1, -1]], dtype=np.int32)
    n_slots = 12
    for free, want in (([7, 6, 4], fresh), ([7], [0, 0, 0])):
        t, _ = run_tables(ek, held, fresh, m=m, n_slots=n_slots, table=table, ps=4, pages_held=[1, 2, 0], free=free, n_pages=8)
        assert t.granted.tolist() == want and t.result[0] == (0 if any(want) else ek.ERR_NO_PAGES)
    for max_ctx, want in ((11, fresh), (10, [0, 0, 0])):
        t, _ = run_tables(ek, held, fresh, m=m, n_slots=n_slots, max_ctx=max_ctx)
        assert t.granted.tolist() == want
    # a caller without the member
    t.desc.granted = None
    t.granted.fill_(-9)
    plane = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    cache = ek.make_cache(plane, plane, n_seqs=3, max_ctx=11)
    ek.elitekv_step_tables(cache, t)
    assert t.granted.tolist() == [-9] * 3 and t.seq_lens.tolist() == [7, 11, 0]
    for same in (t._inputs["held"], t._inputs["fresh"]):
        t.desc.granted = same.data_ptr()
        with pytest.raises(ek.ElitekvError):
            ek.elitekv_step_tables(cache, t)


class Granted(Loop):
    """The loop whose attention and acceptance take what the tables granted."""

    def step(self):
        ek, B, m, w, t = self.ek, self.B, self.m, self.w, self.t
        ek.elitekv_step_tables(self.cache, t)
        ek.elitekv_append_slots(self.layer, self.cache, self.k_e, self.c, t.slot, t.pos)
        ek.elitekv_absorb_query(self.layer, self.q, t.pos, self.q_rope, self.q_abs)
        ek.elitekv_attend_tree(self.layer, self.cache, self.q_rope.view(B, m, w.n_h, -1), self.q_abs.view(B, m, w.n_h, -1), t.seq_lens, t.granted,
                               t.tree_mask, self.ws, self.out)
        ek.elitekv_accept_tree(self.layer, self.cache, self.held, t.granted, self.parent, self.draft, self.first, self.chosen, self.n_acc, self.path,
                               self.first, self.held)
        self.pages.copy_(t.pages_held_out)
        self.n_free.copy_(t.n_free_out)

    def tokens(self, seed, fresh, tree):
        """Queries, keys and drafts of a step; the model confirms each node's lowest child, of two roots the first alone."""
        B, m = self.B, self.m
        g = torch.Generator(device="cpu").manual_seed(seed)
        for x in (self.k_e, self.c, self.q):
            x.copy_(torch.randn(x.shape, generator=g))
        draft = np.random.default_rng(seed).integers(1, 9, (B, m))
        draft[:, 0] = self.first.tolist()
        i = np.arange(m)
        parent = np.tile({"chain": i - 1, "two roots": np.maximum(i - 2, -1), "fork": np.where(i > 1, i - 2, i - 1)}[tree], (B, 1))
        chosen = np.zeros((B, m), dtype=np.int64)
        for i in range(m - 1, 0, -1):
            chosen[np.arange(B), np.maximum(parent[:, i], 0)] = draft[:, i]
        chosen[:, m - 1] = 5
        for to, v in ((self.fresh, fresh), (self.parent, parent), (self.draft, draft), (self.chosen, chosen)):
            to.copy_(i32(v))

    def state(self):
        return [x.clone() for x in (self.rope.view(torch.int16), self.lat.view(torch.int16), self.table, self.held, self.first, self.pages, self.n_free)]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("tree,least", [("chain", 6), ("two roots", 1), ("fork", 3)])
@pytest.mark.parametrize("w,d_ck", [(gen.TINY, 0), (gen.LLAMA7B_75, 512)])
def test_a_refused_step_leaves_everything_as_it_was(ek, w, d_ck, tree, least, graph):
    """A step with too few pages and one with more drafts than fit, between others: every row, length, page and token stays, the
    attention is zero, and the steps behind them give the bits of a loop in which they never were."""
    B, m, ps, held, fresh = 3, 7, 16, [21, 5, 48], [7, 6, 7]
    loops = [Granted(ek, w, B, m, held, ps, seed=4, d_ck=d_ck) for _ in range(2)]
    replay = []
    for lp in loops:
        g = torch.Generator(device="cpu").manual_seed(9)
        lp.prompt([torch.randn((sum(held), *x.shape[1:]), generator=g).to(torch.bfloat16).cuda() for x in (lp.k_e, lp.c)])
        lp.tokens(1, fresh, tree)
        lp.step()
        torch.cuda.synchronize()
        assert lp.t.result[0] == 0 and lp.t.granted.tolist() == fresh and lp.n_acc.min() >= least
        cg = None
        if graph:
            cg = torch.cuda.CUDAGraph()
            with torch.cuda.graph(cg):
                lp.step()
        replay.append(cg.replay if graph else lp.step)
    lp = loops[0]
    # after the chain's first step the next one needs pages, after the others' it fits the pages held
    for kind in ("no pages", "too long")[tree != "chain":]:
        lp.tokens(2, fresh if kind == "no pages" else [7, m + 1, 1], tree)
        n_free = lp.n_free.clone()
        if kind == "no pages":
            lp.n_free.zero_()
        lp.out.fill_(7.0)
        was = lp.state()
        replay[0]()
        torch.cuda.synchronize()
        assert lp.t.result[0] == (ek.ERR_NO_PAGES if kind == "no pages" else ek.ERR_BAD_POSITION) and lp.t.granted.tolist() == [0] * B
        for x, y in zip(lp.state(), was):
            assert torch.equal(x, y)
        assert not lp.out.any() and not lp.n_acc.any() and (lp.path == -1).all()
        assert ek.elitekv_check_status(lp.layer) == 0
        lp.n_free.copy_(n_free)
    for seed in (3, 4):
        for lp, step in zip(loops, replay):
            lp.tokens(seed, fresh, tree)
            step()
        torch.cuda.synchronize()
        for x, y in zip(loops[0].state() + [loops[0].out, loops[0].path], loops[1].state() + [loops[1].out, loops[1].path]):
            assert torch.equal(x, y)
        assert loops[0].t.result[0] == 0 and loops[0].n_acc.min() >= least and ek.elitekv_check_status(loops[0].layer) == 0


# ------------------------------------------------------------------------------- no page is free
@pytest.mark.parametrize("m", [0, 4])
def test_an_empty_stack(ek, m):
    """A pool whose pages are all given out (an empty tensor has no address): steps that need none are granted, others
    refused."""
    table, none = i32([[2, 3], [1, 0]]), torch.empty(0, dtype=torch.int32, device="cuda")
    plane = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    cache = ek.make_cache(plane, plane, n_seqs=2, page_table=table, page_size=4)
    cache.num_pages = 4
    for pages, code, detail in (([2, 2], 0, 0), ([2, 1], ek.ERR_NO_PAGES, 1)):
        t = ek.make_tables(2, 8, m, i32([3, 4]), i32([4, 2]), page_table=table, pages_held=i32(pages), free_pages=none, n_free=i32([0]))
        ek.elitekv_step_tables(cache, t)
        assert t.result.tolist() == [code, 6 if code == 0 else 0, 0, detail] and t.granted.tolist() == ([4, 2] if code == 0 else [0, 0])
        slots = [11, 12, 13, 14] + ([0, 1, -1, -1] if code == 0 else [])
        assert t.slot.tolist() == (slots if code == 0 else [-1] * 8)
        assert t.n_free_out.tolist() == [0] and t.pages_held_out.tolist() == pages and table.tolist() == [[2, 3], [1, 0]]
