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
