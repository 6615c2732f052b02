"""Speculative decoding with a tree of drafted tokens over the compressed cache, as cases that can be timed and compared.

Four operators, in the order in which a serving step uses them:

  kind    "tables"  block table, slot map, rotary positions and tree masks of a step, from lengths
                    (elitekv_step_tables)
          "append"  rotated keys and latents of new tokens into the rows that a slot map names
                    (elitekv_append_slots)
          "tree"    attention of the drafted nodes over the cache: every node sees the committed tokens,
                    its ancestors and itself (elitekv_attend_tree)
          "accept"  the longest branch that the model confirms becomes part of the sequence: its rows
                    move to consecutive slots (elitekv_accept_tree)

`run` computes them with elementary torch operations, or (`own`) through the library's entry points.
Layer shapes are the library's own (paper_2503_01586_b200.inputs), written out here because the plain
forms do not import the package.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
BASE = 10000.0

# name: heads, head dim, elite chunks per head, latent width, model width, width of the key latent (0: joint)
LAYERS = {
    "tiny": (4, 64, 2, 64, 256, 0),
    "7b-75": (32, 128, 8, 1536, 4096, 0),
    "13b-75": (40, 128, 8, 1920, 5120, 0),
    "7b-87.5": (32, 128, 4, 768, 4096, 0),
    "7b-75-slrd": (32, 128, 8, 1536, 4096, 512),
}


def _tree(name, layer, B, ctx, m, ctx_lo=None, paged=False, page_size=64, lens_seed=0):
    case = {"kind": "tree", "layer": layer, "B": B, "ctx": ctx, "ctx_lo": ctx if ctx_lo is None else ctx_lo, "m": m,
            "paged": paged, "page_size": page_size, "lens_seed": lens_seed}
    return case if name is None else {"name": name, **case}


def _tables(name, B, ctx, fresh, tree, page_size=64, lens_seed=0):
    case = {"kind": "tables", "B": B, "ctx": ctx, "fresh": fresh, "tree": tree, "page_size": page_size, "lens_seed": lens_seed}
    return case if name is None else {"name": name, **case}


def _append(name, layer, B, ctx, fresh, tree, page_size=64, lens_seed=0):
    case = {"kind": "append", "layer": layer, "B": B, "ctx": ctx, "fresh": fresh, "tree": tree, "page_size": page_size,
            "lens_seed": lens_seed}
    return case if name is None else {"name": name, **case}


def _accept(name, layer, B, ctx, m, paged=True, page_size=64, lens_seed=0):
    case = {"kind": "accept", "layer": layer, "B": B, "ctx": ctx, "m": m, "paged": paged, "page_size": page_size,
            "lens_seed": lens_seed}
    return case if name is None else {"name": name, **case}


def listed():
    return [
        # the smallest model configuration, one sequence, a small tree of odd size: launches and latency only
        _tree("tree-tiny-b1-ctx201-m7", "tiny", 1, 201, 7),
        # one interactive user of a 7B layer, odd context
        _tree("tree-7b-b1-ctx1999-m16", "7b-75", 1, 1999, 16),
        # the headline serving batch with a handful of drafts per sequence: near the memory bound
        _tree("tree-7b-b16-ctx4096-m4", "7b-75", 16, 4096, 4),
        # continuous batching: ragged contexts over shuffled pages, trees of up to 13 nodes
        _tree("tree-7b-paged-b32-ragged-m13", "7b-75", 32, 16384, 13, ctx_lo=512, paged=True, lens_seed=1003),
        # 13B layer (40 heads), half the largest tree: the tensor cores set the pace
        _tree("tree-13b-b8-ctx8192-m32", "13b-75", 8, 8192, 32),
        # separated key and value latents, the largest tree, ragged contexts
        _tree("tree-7b-slrd-b16-ragged-m64", "7b-75-slrd", 16, 4096, 64, ctx_lo=1024, lens_seed=7),
        # a serving batch's draft step: lengths and parents to page table, slots, positions, masks
        _tables("tables-b32-m16", 32, 16384, 16, True, lens_seed=11),
        # a batch of prompts (or prompt chunks) of up to 2048 new tokens, packed, odd counts
        _tables("tables-b64-packed-2048", 64, 16384, 2048, False, lens_seed=12),
        # the drafts of a serving batch enter the cache
        _append("append-7b-b32-m16", "7b-75", 32, 4096, 16, True, lens_seed=13),
        # prompt chunks enter the paged cache through the slot map
        _append("append-7b-b32-packed-1024", "7b-75", 32, 1024, 1024, False, lens_seed=14),
        # verification of a serving batch's trees
        _accept("accept-7b-b16-m16", "7b-75", 16, 500, 16, lens_seed=15),
        # many sequences, the largest trees
        _accept("accept-13b-b200-m64", "13b-75", 200, 300, 64, lens_seed=16),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _elems(layer):
    n_h, _, r, d_c, _, _ = LAYERS[layer]
    return 2 * r * n_h + d_c


MOST_CACHE = 1.2e9       # bytes: the ragged listed tree
MOST_FLOPS = 4.0e11      # the listed tree of 64 nodes


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "tables", "append", "accept"])
    seed = rng.randrange(1 << 20)
    page_size = rng.choice([16, 32, 64, 128])
    if kind == "tables":
        if rng.random() < 0.5:
            return _tables(None, _log_int(rng, 1, 512), _log_int(rng, 64, 32768), rng.randint(1, 64), True, page_size, seed)
        B = _log_int(rng, 1, 256)
        return _tables(None, B, _log_int(rng, 64, 32768), _log_int(rng, 1, min(4096, 131072 // B)), False, page_size, seed)
    layer = rng.choice(["7b-75", "7b-75", "13b-75", "7b-87.5", "7b-75-slrd", "tiny"])
    if kind == "append":
        B = _log_int(rng, 1, 64)
        if rng.random() < 0.5:
            return _append(None, layer, B, _log_int(rng, 16, 2048), rng.randint(1, 64), True, page_size, seed)
        return _append(None, layer, B, _log_int(rng, 16, 1024), _log_int(rng, 1, max(1, 32768 // B)), False, page_size, seed)
    if kind == "accept":
        return _accept(None, layer, _log_int(rng, 1, 200), _log_int(rng, 16, 300), rng.randint(1, 64), rng.random() < 0.7, page_size, seed)
    B, m = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    n_h, _, r, _, _, _ = LAYERS[layer]
    kw, vw = _widths(layer)
    most = min(MOST_CACHE / (2 * _elems(layer) * B), MOST_FLOPS / (2 * m * n_h * (2 * r + kw + vw) * B))
    ctx = _log_int(rng, max(m, 64), int(min(16384, max(most, 100))))
    return _tree(None, layer, B, ctx, m, ctx_lo=max(m, ctx // 8) if rng.random() < 0.6 else ctx, paged=rng.random() < 0.6,
                 page_size=page_size, lens_seed=seed)


# ------------------------------------------------------------------------------- what a case holds
def _widths(layer):
    _, _, _, d_c, _, d_ck = LAYERS[layer]
    return (d_ck, d_c - d_ck) if d_ck else (d_c, d_c)


def _lens(case):
    """Per sequence: committed tokens and new ones (of the case alone, so that the work does not depend on the seed)."""
    rng = random.Random(case["lens_seed"])
    B, kind = case["B"], case["kind"]
    if kind == "tree":
        m = case["m"]
        total = [rng.randint(case["ctx_lo"], case["ctx"]) for _ in range(B)]
        # trees of one batch differ in size; the first is full, so that the padded width is met
        new = [m if b == 0 or case["ctx_lo"] == case["ctx"] else rng.randint((m + 1) // 2, m) for b in range(B)]
        return [t - n for t, n in zip(total, new)], new
    held = [rng.randint(case["ctx"] // 2, case["ctx"]) for _ in range(B)]
    most = case["m"] if kind == "accept" else case["fresh"]
    return held, [most if b == 0 else rng.randint((most + 1) // 2, most) for b in range(B)]


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEVICE)


def _normal(shape, std, g):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEVICE)
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        hi = min(flat.numel(), lo + (1 << 26))
        flat[lo:hi] = torch.randn(hi - lo, generator=g, device=DEVICE) * std
    return out


def _parents(B, m, rng):
    """Node 0 hangs on the committed tokens, every other node on one before it."""
    u = rng.random((B, m))
    p = np.minimum((u * np.arange(m)).astype(np.int64), np.maximum(np.arange(m) - 1, 0))
    p[:, 0] = -1
    return p.astype(np.int32)


def _planes(case, rows, g):
    n_h, _, r, d_c, _, _ = LAYERS[case["layer"]]
    return _normal((rows, n_h * 2 * r), 1.0, g), _normal((rows, d_c), 1.0, g)


def _pages(need, max_pages, spare, rng):
    """Page table of sequences that hold need[b] pages each out of one shuffled pool, and the pool's free pages."""
    total = sum(need)
    perm = rng.permutation(total + spare).astype(np.int32)
    table = np.full((len(need), max_pages), -1, dtype=np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = perm[at:at + k]
        at += k
    return table, perm[total:], total + spare


def _layer(case, s, g, max_pos):
    n_h, d_h, r, d_c, d, d_ck = LAYERS[case["layer"]]
    kw, vw = _widths(case["layer"])
    cpu = np.random.default_rng(case["lens_seed"] + 5)
    s["elite"] = np.stack([cpu.permutation(d_h // 2)[:r] for _ in range(n_h)]).astype(np.int32)
    s["W_uv"] = _normal((vw, n_h * d_h), d ** -0.5, g)
    theta = BASE ** (-2.0 * torch.arange(d_h // 2, dtype=torch.float64, device=DEVICE) / d_h)
    a = torch.arange(max_pos, dtype=torch.float64, device=DEVICE)[:, None] * theta
    s["cos_sin"] = torch.stack([a.cos(), a.sin()], -1).to(torch.float32)
    s["elite_dev"] = torch.from_numpy(s["elite"]).to(DEVICE).long()
    if own:
        from paper_2503_01586_b200 import binding as ek
        # no call here reads W_uk: numbers of a generator of its own, so that the inputs are the same either way
        W_uk = _normal((kw, n_h * (d_h - 2 * r)), d ** -0.5, torch.Generator(device=DEVICE))
        s["layer"] = ek.Layer(n_h, d_h, r, d_c, torch.from_numpy(s["elite"]), W_uk, s["W_uv"], max_pos, cos_sin=s["cos_sin"], d_ck=d_ck)


def _cache(case, s, B, max_ctx):
    if own:
        from paper_2503_01586_b200 import binding as ek
        s["cache"] = ek.make_cache(s["rope"], s["latent"], n_seqs=B, max_ctx=max_ctx, page_table=s["page_table"],
                                   page_size=case["page_size"])


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    held, new = _lens(case)
    B, kind = case["B"], case["kind"]
    s = {"case": case, "page_table": None, "max_ctx": 0}
    if kind == "tables":
        return _prepare_tables(case, s, held, new, rng)
    ps = case["page_size"]
    total = [h + n for h, n in zip(held, new)]
    max_ctx = max(total) + 1
    if case.get("paged", True):
        need = [(t + ps - 1) // ps for t in total]
        table, _, n_pages = _pages(need, max(need), 0, rng)
        s["page_table"] = torch.from_numpy(table).to(DEVICE)
        rows = n_pages * ps
    else:
        s["max_ctx"], rows = max_ctx, B * max_ctx
    _layer(case, s, g, max_ctx)
    s["rope"], s["latent"] = _planes(case, rows, g)
    _cache(case, s, B, max_ctx)
    s["held"], s["new"] = _ints(held), _ints(new)
    return {"tree": _prepare_tree, "append": _prepare_append, "accept": _prepare_accept}[kind](case, s, held, new, g, rng)


def _prepare_tree(case, s, held, new, g, rng):
    n_h, d_h, r, d_c, d, _ = LAYERS[case["layer"]]
    B, m = case["B"], case["m"]
    kw, _ = _widths(case["layer"])
    s["seq_lens"] = s["held"] + s["new"]
    s["mask"] = _bits(_closure(torch.from_numpy(_parents(B, m, rng)).to(DEVICE)))
    # an absorbed query is a product of d_h - 2r query dims, N(0, 1), with weights N(0, 1/d)
    s["q_abs"] = _normal((B, m, n_h, kw), math.sqrt((d_h - 2 * r) / d), g)
    s["q_rope"] = _normal((B, m, n_h, 2 * r), 1.0, g)
    if own:
        from paper_2503_01586_b200 import binding as ek
        s["workspace"] = torch.empty(ek.elitekv_attend_tree_workspace_size(s["layer"], B, m), dtype=torch.uint8, device=DEVICE)
        s["out"] = torch.empty((B, m, n_h, d_h), dtype=torch.bfloat16, device=DEVICE)
    return s


def _prepare_append(case, s, held, new, g, rng):
    n_h, _, r, d_c, _, _ = LAYERS[case["layer"]]
    B, most, ps = case["B"], case["fresh"], case["page_size"]
    p = torch.arange(most, device=DEVICE)[None] + s["held"][:, None]
    row = _rows(s, p.clamp(max=int(max(h + n for h, n in zip(held, new))) - 1))
    valid = torch.arange(most, device=DEVICE)[None] < s["new"][:, None]
    if case["tree"]:        # the padded batch, as elitekv_step_tables lays it out
        depth = _closure(torch.from_numpy(_parents(B, most, rng)).to(DEVICE)).sum(-1) - 1
        s["slot"] = torch.where(valid, row, -1).reshape(-1)
        s["pos"] = torch.where(valid, s["held"][:, None] + depth, 0).to(torch.int32).reshape(-1)
    else:
        s["slot"], s["pos"] = row[valid], p[valid].to(torch.int32)
    T = s["slot"].numel()
    s["k_e"], s["c"] = _normal((T, n_h, r, 2), 1.0, g), _normal((T, d_c), 1.0, g)
    return s


def _prepare_accept(case, s, held, new, g, rng):
    B, m = case["B"], case["m"]
    parent = _parents(B, m, rng)
    draft = rng.integers(0, 32000, (B, m)).astype(np.int32)
    chosen = rng.integers(0, 32000, (B, m)).astype(np.int32)
    for b in range(B):                  # the draft model is right about two times out of three
        for i in range(1, m):
            if rng.random() < 0.66:
                chosen[b, parent[b, i]] = draft[b, i]
    s["parent"], s["draft"], s["chosen"] = (torch.from_numpy(x).to(DEVICE) for x in (parent, draft, chosen))
    s["first"] = s["draft"][:, 0].contiguous()
    s["n_accepted"], s["token"], s["held_out"] = (torch.empty(B, dtype=torch.int32, device=DEVICE) for _ in range(3))
    s["path"] = torch.empty((B, m), dtype=torch.int32, device=DEVICE)
    return s


def _prepare_tables(case, s, held, new, rng):
    B, ps, most = case["B"], case["page_size"], case["fresh"]
    # pages of the last step's drafts stay with their sequence: some hold one more than their tokens need
    kept = random.Random(case["lens_seed"] + 1)
    pages = [(h + ps - 1) // ps + int(kept.random() < 0.3) for h in held]
    max_pages = max(p + (n + ps - 1) // ps + 1 for p, n in zip(pages, new))
    table, free, n_pages = _pages(pages, max_pages, sum((n + ps - 1) // ps + 1 for n in new) + 5, rng)
    m = most if case["tree"] else 0
    n_slots = B * m if m else sum(new) + 3
    s |= {"page_table": torch.from_numpy(table).to(DEVICE), "held": _ints(held), "new": _ints(new), "pages_held": _ints(pages),
          "free_pages": torch.from_numpy(free.copy()).to(DEVICE), "n_free": _ints([len(free)]), "m": m, "n_slots": n_slots,
          "parent": torch.from_numpy(_parents(B, m, rng)).to(DEVICE) if m else None}
    if own:
        from paper_2503_01586_b200 import binding as ek
        # the planes are not touched by the tables: a descriptor of the pool is enough
        s["planes"] = torch.zeros((n_pages * ps, 8), dtype=torch.bfloat16, device=DEVICE)
        s["cache"] = ek.make_cache(s["planes"], s["planes"], n_seqs=B, page_table=s["page_table"], page_size=ps)
        s["tables"] = ek.make_tables(B, s["n_slots"], m, s["held"], s["new"], parent=s["parent"], page_table=s["page_table"],
                                     pages_held=s["pages_held"], free_pages=s["free_pages"], n_free=s["n_free"])
    return s


# ------------------------------------------------------------------------------- plain forms
def _closure(parent):
    """[B][m][m] truth values: node j is node i itself or one of its ancestors."""
    B, m = parent.shape
    i = torch.arange(m, device=parent.device)
    step = (parent[:, :, None] == i) | (i[:, None] == i)
    # (1 + N)^64 holds the binomial coefficient of the distance wherever a path of up to 64 steps leads
    return torch.linalg.matrix_power(step.double(), 64) > 0.5


def _bits(closure):
    return (closure.long() << torch.arange(closure.shape[-1], device=closure.device)).sum(-1)


def _rows(s, p):
    """Plane row of position p [B][n] of every sequence."""
    ps, B = s["case"]["page_size"], p.shape[0]
    if s["page_table"] is None:
        return p.long() + torch.arange(B, device=p.device)[:, None] * s["max_ctx"]
    return torch.gather(s["page_table"], 1, (p // ps).long()).long() * ps + p % ps


def _tree_plain(s):
    case = s["case"]
    n_h, d_h, r, d_c, _, _ = LAYERS[case["layer"]]
    B, m = case["B"], case["m"]
    kw, vw = _widths(case["layer"])
    n = case["ctx"]
    t = torch.arange(n, device=DEVICE)[None].expand(B, n)
    row = _rows(s, torch.minimum(t, s["seq_lens"][:, None] - 1))
    k = s["rope"][row].float().view(B, n, n_h, 2 * r)
    c = s["latent"][row].float()
    score = torch.einsum("bihd,bthd->biht", s["q_rope"].float(), k)
    score += (s["q_abs"].float().view(B, m * n_h, kw) @ c[..., :kw].transpose(1, 2)).view(B, m, n_h, n)
    node = t - s["held"][:, None]                       # < 0: committed
    seen = (s["mask"][:, :, None] >> node.clamp(0, 63)[:, None] & 1).bool() | (node < 0)[:, None]
    seen = seen & (t < s["seq_lens"][:, None])[:, None]
    seen = seen & (torch.arange(m, device=DEVICE)[None] < s["new"][:, None])[:, :, None]
    score = score.mul_(d_h ** -0.5).masked_fill_(~seen[:, :, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == float("-inf"), 0.0, top))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    o = (p.reshape(B, m * n_h, n) @ c[..., -vw:]).view(B, m, n_h, vw)
    return torch.einsum("bihv,vhd->bihd", o, s["W_uv"].float().view(vw, n_h, d_h)).to(torch.bfloat16)


def _append_plain(s):
    n_h, d_h, r, d_c, _, _ = LAYERS[s["case"]["layer"]]
    on = s["slot"] >= 0
    at = torch.where(on, s["slot"], s["slot"].max())          # padding writes what its row holds anyway
    cs = s["cos_sin"][s["pos"].long()[:, None, None], s["elite_dev"][None]]
    x, y = s["k_e"].float().unbind(-1)
    rot = torch.stack([x * cs[..., 0] - y * cs[..., 1], x * cs[..., 1] + y * cs[..., 0]], -1).to(torch.bfloat16).view(-1, n_h * 2 * r)
    last = torch.argmax(s["slot"])
    s["rope"][at] = torch.where(on[:, None], rot, rot[last][None])
    s["latent"][at] = torch.where(on[:, None], s["c"], s["c"][last][None])
    return s["rope"], s["latent"]


def _accept_plain(s):
    B, m = s["parent"].shape
    parent, i = s["parent"].long(), torch.arange(m, device=DEVICE)
    want = torch.where(parent < 0, s["first"][:, None], torch.gather(s["chosen"], 1, parent.clamp(min=0)))
    ok = (s["draft"] == want) & (i < s["new"][:, None])
    # the lowest of several fitting children
    same = (parent[:, :, None] == parent[:, None, :]) & ok[:, None, :] & (i[None, :] < i[:, None])
    ok = ok & ~same.any(-1)
    taken = ~(_closure(s["parent"]) & ~ok[:, None, :]).any(-1)
    count = taken.sum(-1)
    order = torch.argsort(torch.where(taken, i, i + m), dim=1)          # accepted nodes first, ascending
    path = torch.where(i < count[:, None], order, -1)
    end = torch.gather(path, 1, (count - 1).clamp(min=0)[:, None])[:, 0]
    token = torch.where(count > 0, torch.gather(s["chosen"], 1, end.clamp(min=0)[:, None])[:, 0], s["first"])
    own_place = torch.minimum(i, s["new"][:, None] - 1)
    dst = _rows(s, s["held"][:, None] + own_place)
    src = _rows(s, s["held"][:, None] + torch.where(path < 0, own_place, path))
    # a row past a sequence's nodes is its last node's row, which keeps what that node's own place gets
    src = torch.where(i < s["new"][:, None], src, torch.gather(src, 1, (s["new"][:, None] - 1).long()))
    for plane in (s["rope"], s["latent"]):
        plane[dst.view(-1)] = plane[src.view(-1)]
    i32 = torch.int32
    return {"n_accepted": count.to(i32), "path": path.to(i32), "token": token, "held": (s["held"] + count).to(i32),
            "rope": s["rope"], "latent": s["latent"]}


def _tables_plain(s):
    B, ps, m, n_slots = s["case"]["B"], s["case"]["page_size"], s["m"], s["n_slots"]
    held, new, ph = s["held"].long(), s["new"].long(), s["pages_held"].long()
    need = ((held + new + ps - 1) // ps - ph).clamp(min=0)
    before = need.cumsum(0) - need
    col = torch.arange(s["page_table"].shape[1], device=DEVICE)[None] - ph[:, None]
    k = (s["n_free"].long() - 1 - before[:, None] - col).clamp(0, s["free_pages"].numel() - 1)
    s["page_table"].copy_(torch.where((col >= 0) & (col < need[:, None]), s["free_pages"][k], s["page_table"]))
    first = torch.cat([held.new_zeros(1), new.cumsum(0)])
    t = torch.arange(n_slots, device=DEVICE)
    if m:
        b, i = t // m, t % m
        on = i < new[b]
    else:
        b = torch.searchsorted(first[1:].contiguous(), t, right=True).clamp(max=B - 1)
        i = t - first[b]
        on = t < first[-1]
    p = torch.where(on, held[b] + i, 0)
    slot = s["page_table"][b, p // ps].long() * ps + p % ps
    i32 = torch.int32
    out = {"page_table": s["page_table"], "pages_held": (ph + need).to(i32), "n_free": (s["n_free"] - need.sum()).to(i32),
           "seq_lens": (held + new).to(i32), "first": first.to(i32), "seq_id": torch.where(on, b, -1).to(i32),
           "slot": torch.where(on, slot, -1),
           "result": torch.stack([need.new_zeros(()), first[-1], need.sum(), need.new_zeros(())]).to(i32)}
    if m:
        line = _closure(s["parent"])
        real = torch.arange(m, device=DEVICE) < new[:, None]
        out["pos"] = torch.where(real, held[:, None] + line.sum(-1) - 1, 0).to(i32).view(-1)
        out["tree_mask"] = torch.where(real, _bits(line), 0)
    else:
        out["pos"] = p.to(i32)
    return out


# ------------------------------------------------------------------------------- one pass
def _run_own(s):
    from paper_2503_01586_b200 import binding as ek
    kind = s["case"]["kind"]
    if kind == "tree":
        return ek.elitekv_attend_tree(s["layer"], s["cache"], s["q_rope"], s["q_abs"], s["seq_lens"], s["new"], s["mask"],
                                      s["workspace"], s["out"])
    if kind == "append":
        ek.elitekv_append_slots(s["layer"], s["cache"], s["k_e"], s["c"], s["slot"], s["pos"])
        return s["rope"], s["latent"]
    if kind == "accept":
        ek.elitekv_accept_tree(s["layer"], s["cache"], s["held"], s["new"], s["parent"], s["draft"], s["first"], s["chosen"],
                               s["n_accepted"], s["path"], s["token"], s["held_out"])
        return {"n_accepted": s["n_accepted"], "path": s["path"], "token": s["token"], "held": s["held_out"],
                "rope": s["rope"], "latent": s["latent"]}
    t = s["tables"]
    ek.elitekv_step_tables(s["cache"], t)
    out = {"page_table": s["page_table"], "pages_held": t.pages_held_out, "n_free": t.n_free_out, "seq_lens": t.seq_lens,
           "first": t.first, "seq_id": t.seq_id, "slot": t.slot, "pos": t.pos, "result": t.result}
    if s["m"]:
        out["tree_mask"] = t.tree_mask
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"tree": _tree_plain, "append": _append_plain, "accept": _accept_plain, "tables": _tables_plain}[state["case"]["kind"]](state)


# ------------------------------------------------------------------------------- floors
def work(case):
    held, new = _lens(case)
    B, kind = case["B"], case["kind"]
    if kind == "tables":
        tokens = case["B"] * case["fresh"] if case["tree"] else sum(new)
        pages = sum((n + case["page_size"] - 1) // case["page_size"] for n in new)
        # lengths in and out, parents in, slot (8), position, sequence (4 each), mask (8) out, page ids in and out
        return {"bytes": 32 * B + tokens * (16 + (12 if case["tree"] else 0)) + 8 * pages, "flops": 0}
    n_h, d_h, r, d_c, _, _ = LAYERS[case["layer"]]
    row = 2 * _elems(case["layer"])
    if kind == "append":
        return {"bytes": sum(new) * (2 * row + 12), "flops": sum(new) * n_h * r * 6}
    if kind == "accept":
        # about half of a path's rows move, once in and once out; lists in and out
        return {"bytes": B * (2 * row + 16 * case["m"] + 24), "flops": 0}
    kw, vw = _widths(case["layer"])
    nodes = sum(new)
    return {"bytes": sum(h + n for h, n in zip(held, new)) * row + nodes * n_h * 2 * (kw + 2 * r + d_h) + 2 * vw * n_h * d_h,
            "flops": sum(n * (h + n) for h, n in zip(held, new)) * n_h * 2 * (2 * r + kw + vw) + nodes * n_h * 2 * vw * d_h}


# ------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    kind = case["kind"]
    if kind == "tables" or work(case)["flops"] > 5e11:
        return None
    s = prepare(case, seed)
    if kind == "append":
        return _append_exact(s)
    if kind == "accept":
        return _accept_exact(s)
    n_h, d_h, r, d_c, _, _ = LAYERS[case["layer"]]
    kw, vw = _widths(case["layer"])
    held, new = _lens(case)
    W = s["W_uv"].double().view(vw, n_h, d_h).transpose(0, 1)
    out = torch.zeros((case["B"], case["m"], n_h, d_h), dtype=torch.float64, device=DEVICE)
    for b, (h, k) in enumerate(zip(held, new)):
        n = h + k
        if case["paged"]:
            ps = case["page_size"]
            at = torch.cat([torch.arange(p * ps, p * ps + ps) for p in s["page_table"][b].tolist()[:(n + ps - 1) // ps]])[:n].to(DEVICE)
        else:
            at = torch.arange(b * s["max_ctx"], b * s["max_ctx"] + n, device=DEVICE)
        lat, rope = s["latent"][at].double(), s["rope"][at].double().view(n, n_h, 2 * r)
        hide = torch.zeros((k, n), dtype=torch.bool)
        for i, bits in enumerate(s["mask"][b, :k].tolist()):
            for j in range(k):
                hide[i, h + j] = not bits >> j & 1
        for hd in range(n_h):
            z = s["q_rope"][b, :k, hd].double() @ rope[:, hd].T + s["q_abs"][b, :k, hd].double() @ lat[:, :kw].T
            z = (z / math.sqrt(d_h)).masked_fill(hide.to(DEVICE), -math.inf)
            out[b, :k, hd] = torch.softmax(z, -1) @ lat[:, d_c - vw:] @ W[hd]
    return out


def _append_exact(s):
    n_h, d_h, r, _, _, _ = LAYERS[s["case"]["layer"]]
    rope, latent = s["rope"].double(), s["latent"].double()
    keep = s["slot"] >= 0
    at, pos = s["slot"][keep], s["pos"][keep].double()
    z = torch.view_as_complex(s["k_e"][keep].double().contiguous())
    turn = pos[:, None, None] * BASE ** (-2.0 * s["elite_dev"].double() / d_h)
    rope[at] = torch.view_as_real(z * torch.polar(torch.ones_like(turn), turn)).reshape(at.numel(), -1)
    latent[at] = s["c"][keep].double()
    return rope, latent


def _accept_exact(s):
    rope, latent = s["rope"].double(), s["latent"].double()
    held, new = _lens(s["case"])
    par, draft, chosen, first = (s[k].tolist() for k in ("parent", "draft", "chosen", "first"))
    ps = s["case"]["page_size"]
    table = s["page_table"].tolist() if s["page_table"] is not None else None
    src, dst = [], []
    for b, (h, k) in enumerate(zip(held, new)):
        where = [(table[b][(h + i) // ps] * ps + (h + i) % ps) if table else b * s["max_ctx"] + h + i for i in range(k)]
        at, want, n = -1, first[b], 0
        for i in range(k):
            if par[b][i] == at and draft[b][i] == want:
                src.append(where[i])
                dst.append(where[n])
                at, want, n = i, chosen[b][i], n + 1
    src, dst = _ints(src, torch.int64), _ints(dst, torch.int64)
    rope[dst], latent[dst] = rope[src], latent[src]
    return {"n_accepted": None, "path": None, "token": None, "held": None, "rope": rope, "latent": latent}
