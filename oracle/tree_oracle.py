"""Float64 CPU oracle of decoding with a tree of drafted tokens (the tables of a step, the attention of a tree over the
compressed cache, greedy acceptance).  TEST INFRASTRUCTURE ONLY: plain loops, no code shared with the CUDA path.

A tree's node i follows node parent[i] < i, or the committed tokens (any other value); it lies in the cache at
position held + i and was rotated at position held + depth(i)."""
from __future__ import annotations

import numpy as np

F64 = np.float64


def real_parent(parent, i):
    p = i - 1 if parent is None else int(parent[i])
    return p if 0 <= p < i else -1


def ancestors(parent, i):
    """Node i and the nodes above it."""
    out = [i]
    while (i := real_parent(parent, i)) >= 0:
        out.append(i)
    return out


def mask_bits(parent, n):
    return [sum(1 << j for j in ancestors(parent, i)) for i in range(n)]


def step_tables(held, fresh, *, m, n_slots, parent=None, page_table=None, page_size=64, pages_held=None, free_pages=None, max_ctx=None):
    """Everything that elitekv_step_tables writes, as a dict (a step that fits).  page_table [B][max_pages]."""
    B = len(held)
    out = {"seq_id": [-1] * n_slots, "pos": [0] * n_slots, "slot": [-1] * n_slots, "seq_lens": [], "first": [0], "pages_held": []}
    table = None if page_table is None else np.array(page_table)
    stack = None if page_table is None else list(free_pages)
    if m:
        out["tree_mask"] = np.zeros((B, m), dtype=np.uint64)
    taken = 0
    for b in range(B):
        n = held[b] + fresh[b]
        if table is not None:
            have = pages_held[b]
            while have * page_size < n:
                table[b, have] = stack.pop()
                have += 1
                taken += 1
            out["pages_held"].append(have)
        for i in range(fresh[b]):
            at = b * m + i if m else out["first"][b] + i
            p = held[b] + i
            out["seq_id"][at] = b
            out["slot"][at] = b * max_ctx + p if table is None else int(table[b, p // page_size]) * page_size + p % page_size
            out["pos"][at] = p
            if m:
                line = ancestors(None if parent is None else parent[b], i)
                out["pos"][at] = held[b] + len(line) - 1
                out["tree_mask"][b, i] = sum(1 << j for j in line)
        out["seq_lens"].append(n)
        out["first"].append(out["first"][b] + fresh[b])
    out["page_table"] = table
    out["n_free"] = None if stack is None else len(stack)
    out["result"] = [0, out["first"][-1], taken, 0]
    return out


def attend_tree(q_rope, q_abs, k_rope, c_k, c_v, W_uv, prefix, bits, scale):
    """One sequence.  q_rope [k][n_h][2r], q_abs [k][n_h][kw], k_rope [n][n_h][2r], c_k [n][kw], c_v [n][vw],
    W_uv [vw][n_h * d_h], bits: the k nodes' masks.  Returns [k][n_h][d_h].  What a row does not see is not touched."""
    k, n_h, _ = q_abs.shape
    d_h = W_uv.shape[1] // n_h
    out = np.zeros((k, n_h, d_h), dtype=F64)
    n = c_k.shape[0]
    for i in range(k):
        seen = [t for t in range(n) if t < prefix or int(bits[i]) >> (t - prefix) & 1]
        if not seen:
            continue
        for h in range(n_h):
            s = scale * (k_rope[seen, h] @ q_rope[i, h] + c_k[seen] @ q_abs[i, h])
            p = np.exp(s - s.max())
            out[i, h] = (p @ c_v[seen] / p.sum()) @ W_uv[:, h * d_h:(h + 1) * d_h]
    return out


def accept(parent, draft, first, chosen, n):
    """(accepted nodes in order, the choice after them) of one sequence."""
    at, want, path = -1, int(first), []
    while True:
        fit = [i for i in range(n) if real_parent(parent, i) == at and int(draft[i]) == want and i > at]
        if not fit:
            return path, want
        at = fit[0]
        path.append(at)
        want = int(chosen[at])
