"""Sizes that the binding of the tree calls refuses before anything reaches the library (no GPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2503_01586_b200 import binding as ek

LAYER = SimpleNamespace(handle=None, n_h=2, r=2, d_c=8, d_h=16, kw=8)


def zeros(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype)


def refused(fn, good, **bad):
    for k, v in bad.items():
        with pytest.raises(ValueError):
            fn(LAYER, None, **(good | {k: v}))


def test_sizes_of_append_slots():
    bf16 = torch.bfloat16
    good = {"k_e": zeros(5, 2, 2, 2, dtype=bf16), "c": zeros(5, 8, dtype=bf16), "slot": zeros(5, dtype=torch.int64), "pos": zeros(5)}
    refused(ek.elitekv_append_slots, good, k_e=zeros(5, 2, 2, dtype=bf16), c=zeros(5, 7, dtype=bf16), slot=zeros(4, dtype=torch.int64), pos=zeros(4))


def test_sizes_of_attend_tree():
    bf16 = torch.bfloat16
    good = {"q_rope": zeros(3, 4, 2, 4, dtype=bf16), "q_abs": zeros(3, 4, 2, 8, dtype=bf16), "seq_lens": zeros(3), "n_nodes": zeros(3),
            "tree_mask": zeros(3, 4, dtype=torch.int64), "workspace": None, "out": zeros(3, 4, 2, 16, dtype=bf16)}
    refused(ek.elitekv_attend_tree, good, q_rope=zeros(3, 4, 2, 2, dtype=bf16), q_abs=zeros(3, 3, 2, 8, dtype=bf16), seq_lens=zeros(2),
            n_nodes=zeros(2), tree_mask=zeros(3, 3, dtype=torch.int64), out=zeros(3, 4, 2, 8, dtype=bf16))


def test_sizes_of_accept_tree():
    good = {k: zeros(3) for k in ("held", "n_nodes", "first", "n_accepted", "token", "held_out")} | \
           {k: zeros(3, 4) for k in ("parent", "draft", "chosen", "path")}
    refused(ek.elitekv_accept_tree, good, **{k: zeros(2) for k in ("held", "n_nodes", "first", "n_accepted", "token", "held_out")},
            **{k: zeros(3, 3) for k in ("parent", "draft", "chosen", "path")})
