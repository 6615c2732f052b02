"""A workspace sized for the largest call of tree attention serves the smaller ones."""
import pytest
import torch

from paper_2503_01586_b200 import inputs as gen

from .test_gpu_tree import ODD, call_tree, ek, tree_state  # noqa: F401  (ek is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w,d_ck", [(gen.LLAMA7B_75, 0), (gen.LLAMA13B_75, 0), (gen.LLAMA7B_75, 512), (ODD, 0), (gen.TINY, 0)])
def test_sizes_grow_with_sequences_and_nodes(ek, w, d_ck):
    layer = tree_state(ek, w, [4], [1], 1, d_ck=d_ck)["layer"]
    batches = [*range(1, 17), 64, 300]
    size = {(B, m): ek.elitekv_attend_tree_workspace_size(layer, B, m) for B in batches for m in range(1, 65)}
    for B in batches:
        assert all(size[B, m] >= size[B, m - 1] for m in range(2, 65))
    for B, C in zip(batches, batches[1:]):
        assert all(size[C, m] >= size[B, m] for m in range(1, 65))


@pytest.mark.parametrize("w,B,m", [(gen.LLAMA7B_75, 1, 64), (gen.LLAMA13B_75, 2, 40), (ODD, 9, 12)])
def test_one_workspace_for_all(ek, w, B, m):
    """The bits that a call has in a workspace of its own, and nothing written behind the end."""
    big = None
    for b, k in ((B, m), (1, 33), (1, 42), (1, 7), (B, 1), (1, 1), (1, 16), (B, 2), (max(B - 1, 1), m - 1), (max(B - 2, 1), 4)):
        k = min(k, m)
        s = tree_state(ek, w, [k + 200 + 37 * x for x in range(b)], [k] * b, k, seed=k)
        want = call_tree(ek, s)
        if big is None:
            n = ek.elitekv_attend_tree_workspace_size(s["layer"], B, m)
            big = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        s["ws"] = big[:n]
        assert torch.equal(call_tree(ek, s), want), (b, k)
        assert (big[n:] == 0xA5).all()
