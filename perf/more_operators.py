"""The operators of a step over a tree of drafted tokens: what is measured of
them, and their plain forms.

A drafter that is unsure proposes several continuations at once: a tree whose
root (row 0) is the last committed token x0.  One forward checks all of it,
and the step keeps the path that the verifier agrees with.  A case is a dict
of plain values; ``kind`` names the operator:

  masks    dvs.tree_masks: who is whose ancestor, and how deep, from the parents
  append   dvs.kv_append_rope: queries and keys rotated, keys and values into
           the paged cache
  attn     dvs.attn_tree: attention of the tree's rows over the cache
  commit   dvs.accept_commit_tree: the accepted path, its cache slots moved
           together, tokens and pages committed

``own`` false: elementary torch operations.  ``own`` true: the framework's
calls.  Lengths, tables, trees and accepted paths follow from the case alone;
tokens, queries, keys and values (and, for masks, the trees) from the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
PAGE = 16
THETA = 10000.0
MAX_NEW = 256


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # The trees of one serving step: 64 sequences of 64 drafted rows.
        dict(name="masks_serving", kind="masks", S=64, rows=64, tree="wide", ragged=True),
        # As many rows as a tree may have (a draft block per acceptance of a
        # block of 32 has about as many), ragged, in a large batch.
        dict(name="masks_large", kind="masks", S=128, rows=1000, tree="deep", ragged=True),
        # A decode step's single token of 64 sequences (heads of the 16-layer
        # decoder stack): latency.
        dict(name="append_single_tokens", kind="append", S=64, rows=1, kv_lo=900, kv_hi=4100,
             heads=16, kv_heads=4, head_dim=96, dtype="bf16", rot_dim=96, tree="none"),
        # The prefill of 8 documents, 1024 vision and 64 prompt rows each,
        # from the fused projection's rows.
        dict(name="append_prefill", kind="append", S=8, rows=1088, kv_lo=0, kv_hi=0, heads=16,
             kv_heads=4, head_dim=96, dtype="bf16", rot_dim=96, tree="none"),
        # Trees in single precision, half of each head rotated, an odd number
        # of rows that starts anywhere in a page.
        dict(name="append_tree_odd", kind="append", S=5, rows=37, kv_lo=11, kv_hi=9001, heads=8,
             kv_heads=2, head_dim=64, dtype="f32", rot_dim=32, tree="deep"),
        # One sequence of 2048 cached tokens, 32 rows: latency of a launch.
        dict(name="attn_one_sequence", kind="attn", S=1, rows=32, kv_lo=2048, kv_hi=2048, heads=16,
             kv_heads=4, head_dim=128, dtype="bf16", tree="wide", ragged=False),
        # Ordinary serving: 32 sequences of 1k-8k, 32 rows.
        dict(name="attn_serving", kind="attn", S=32, rows=32, kv_lo=1024, kv_hi=8192, heads=16,
             kv_heads=4, head_dim=128, dtype="bf16", tree="wide", ragged=True),
        # Long documents: 64 sequences of 4k-16k, 64 rows.
        dict(name="attn_long_document", kind="attn", S=64, rows=64, kv_lo=4096, kv_hi=16384,
             heads=16, kv_heads=4, head_dim=128, dtype="bf16", tree="deep", ragged=False),
        # Single tokens (a tree of its root alone) of a ragged batch, small
        # heads.
        dict(name="attn_single_tokens", kind="attn", S=48, rows=1, kv_lo=37, kv_hi=6001, heads=32,
             kv_heads=8, head_dim=64, dtype="bf16", tree="wide", ragged=False),
        # Single precision, an odd number of rows, short caches.
        dict(name="attn_f32_odd", kind="attn", S=4, rows=23, kv_lo=301, kv_hi=2003, heads=8,
             kv_heads=2, head_dim=96, dtype="f32", tree="deep", ragged=True),
        # The commit of a step of the 16-layer stack, 8 sequences of 64 rows.
        dict(name="commit_stack", kind="commit", S=8, rows=64, layers=16, kv_heads=4, head_dim=96,
             dtype="bf16", kv_lo=1088, kv_hi=2112, tree="deep", match=0.85, done=0.0),
        # A large batch of short caches in two layers, some of it finished.
        dict(name="commit_batch", kind="commit", S=64, rows=33, layers=2, kv_heads=4, head_dim=64,
             dtype="f32", kv_lo=20, kv_hi=700, tree="wide", match=0.8, done=0.1),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(16, 4), (8, 2), (32, 8), (8, 4), (12, 2), (4, 4), (16, 1)]


def draw(rng):
    kind = rng.choice(["masks", "append", "append", "attn", "attn", "attn", "attn", "commit"])
    if kind == "masks":
        rows = _log(rng, 8, 1024)
        return dict(kind=kind, S=_log(rng, 1, min(256, max(1, 128000 // rows))), rows=rows,
                    tree=rng.choice(["wide", "deep"]), ragged=True)
    tree = rng.choice(["wide", "deep", "chain"])
    heads, kv_heads = rng.choice(HEADS)
    c = dict(kind=kind, S=_log(rng, 1, 64), rows=_log(rng, 1, 64), heads=heads, kv_heads=kv_heads,
             head_dim=rng.choice([64, 96, 128]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
             tree=tree)
    if kind == "attn":
        c["kv_hi"] = _log(rng, 16, 16384)
        c["ragged"] = rng.random() < 0.6
    elif kind == "append":
        if rng.random() < 0.6:
            c.update(tree="none", rows=_log(rng, 1, 1088))
        c["rot_dim"] = rng.choice([c["head_dim"], c["head_dim"], 32, 0])
        c["kv_hi"] = _log(rng, 16, 16384)
    else:
        del c["heads"]
        c.update(layers=rng.randint(1, 16), kv_hi=_log(rng, 16, 2048),
                 match=round(rng.uniform(0.3, 0.95), 2), done=rng.choice([0.0, 0.0, 0.2]))
    c["kv_lo"] = max(1, c["kv_hi"] // rng.randint(1, 8))
    if kind == "attn" and c["dtype"] == "f32":
        c["kv_hi"] = min(c["kv_hi"], 4096)
        c["kv_lo"] = min(c["kv_lo"], c["kv_hi"])
    # no drawn case costs more than the largest listed ones, nor a larger pool
    top = work(next(x for x in listed() if x["name"] == {
        "append": "append_prefill", "attn": "attn_long_document", "commit": "commit_stack"}[kind]))
    flops = top["flops"] / (12 if c["dtype"] == "f32" else 1)
    while c["S"] > 1 and (work(c)["bytes"] > top["bytes"] or work(c)["flops"] > flops
                          or _pool_bytes(c) > 1.5e9):
        c["S"] = (c["S"] + 1) // 2
    return c


def _es(case):
    return 4 if case["dtype"] == "f32" else 2


def _dt(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lens(case):
    r = random.Random("%d %d %d" % (case["S"], case["kv_lo"], case["kv_hi"]))
    return np.array([r.randint(case["kv_lo"], case["kv_hi"]) for _ in range(case["S"])], np.int64)


def _pool_bytes(case):
    pages = int(-(-(_lens(case) + case["rows"]) // PAGE).sum()) * 1.1
    return pages * case.get("layers", 1) * 2 * case["kv_heads"] * PAGE * case["head_dim"] * _es(case)


def _parents(case, salt=0):
    """[S, rows] parents: -1 for the root, -2 for the padding of a shorter tree.
    wide: levels that grow; deep: mostly runs, some of them branching; chain."""
    S, R = case["S"], case["rows"]
    g = np.random.default_rng([S, R, 11, salt])
    r = np.arange(R)
    if case["tree"] == "chain":
        p = np.broadcast_to(r - 1, (S, R)).copy()
    elif case["tree"] == "wide":
        lo = np.maximum(0, (r - 1) // 4)
        p = lo + (g.random((S, R)) * np.maximum(1, r // 2 - lo)).astype(np.int64)
    else:
        p = np.where(g.random((S, R)) < 0.7, r - 1,
                     (g.random((S, R)) * r).astype(np.int64))
    p[:, 0] = -1
    if case.get("ragged"):
        n = g.integers(max(1, R // 2), R + 1, S)
        p[r[None, :] >= n[:, None]] = -2
    return p.astype(np.int32)


def _paths(case, parents):
    """The rows below the root that each sequence accepts, in order."""
    g = random.Random("%d %d %g" % (case["S"], case["rows"], case["match"]))
    paths = []
    for p in parents:
        at, path = 0, []
        while g.random() < case["match"]:
            children = np.flatnonzero(p == at)
            if not len(children):
                break
            at = int(children[g.randrange(len(children))])
            path.append(at)
        paths.append(path)
    return paths


def _done(case):
    g = random.Random("%d %g" % (case["S"], case["done"]))
    return np.array([g.random() < case["done"] for _ in range(case["S"])])


def work(case):
    S, R = case["S"], case["rows"]
    if case["kind"] == "masks":
        return {"bytes": S * R * (4 + 4 + 4 * ((R + 31) // 32)), "flops": 0}
    row = case["head_dim"] * _es(case)                          # one head's row
    if case["kind"] == "append":
        heads = case["heads"] + 2 * case["kv_heads"]
        return {"bytes": 2 * S * R * heads * row,
                "flops": 3 * S * R * (case["heads"] + case["kv_heads"]) * case["rot_dim"]}
    if case["kind"] == "attn":
        lens = _lens(case)
        # a row multiplies with the cache and its ancestors: at least itself
        return {"bytes": int((lens + R).sum()) * 2 * case["kv_heads"] * row
                + 2 * S * R * case["heads"] * row,
                "flops": 4 * int((lens + 1).sum()) * R * case["heads"] * case["head_dim"]}
    moved = sum(sum(r != i + 1 for i, r in enumerate(p))
                for p, f in zip(_paths(case, _parents(case)), _done(case)) if not f)
    return {"bytes": 2 * moved * 2 * case["layers"] * case["kv_heads"] * row + 12 * S * R, "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _cache(case):
    """Lengths, page table (scattered ids) and free pages, from the case alone."""
    lens, R = _lens(case), case["rows"]
    need = -(-(lens + R) // PAGE)
    width = int(-(-(int(lens.max()) + 2 * R + 1) // PAGE)) + 1
    held = int(need.sum())
    pool = held + case["S"] * (R // PAGE + 2)
    ids = np.random.default_rng([case["S"], R, case["kv_hi"]]).permutation(pool).astype(np.int32)
    table = np.full((case["S"], width), -1, np.int32)
    table[np.arange(width) < need[:, None]] = ids[:held]
    stack = np.full(pool, -1, np.int32)
    stack[:pool - held] = ids[held:]
    return lens.astype(np.int32), table, need.astype(np.int32), stack, pool - held, pool


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _pools(case, pages, g):
    heads, D = case["kv_heads"], case["head_dim"]
    lead = (case["layers"],) if "layers" in case else ()
    return [torch.randn(lead + (pages, heads) + page, device="cuda", generator=g, dtype=_dt(case))
            for page in ((PAGE, D), (D, PAGE))]


def prepare(case, seed):
    if case["kind"] == "masks":
        # the trees are what the call reads: they follow from the seed too
        return dict(case=case, parent=_dev(_parents(case, 1 + seed)))
    lens, table, need, stack, top, pool = _cache(case)
    st = dict(case=case, pools=_pools(case, pool, _gen(seed, 3)))
    S, R, Hq, Hkv, D = (case["S"], case["rows"], case.get("heads"), case["kv_heads"],
                        case["head_dim"])
    if case["kind"] == "commit":
        return _prepare_commit(case, seed, st, lens, table, need, stack, top, pool)
    st.update(table=_dev(table), kv_len=_dev(lens))
    if case["kind"] == "append":
        # the rows of one projection: queries, keys and values side by side
        x = torch.randn((S, R, (Hq + 2 * Hkv) * D), device="cuda", generator=_gen(seed, 1),
                        dtype=_dt(case))
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], dim=-1)
        st.update(q=q.unflatten(-1, (Hq, D)), k=k.unflatten(-1, (Hkv, D)),
                  v=v.unflatten(-1, (Hkv, D)), depth=None)
        if case["tree"] != "none":
            reach = _reach(_dev(_parents(case)))
            st["depth"] = (reach.sum(-1) - 1).to(torch.int32)
    else:
        st["q"] = 2 * torch.randn((S, R, Hq, D), device="cuda", generator=_gen(seed, 1),
                                  dtype=_dt(case))
        st["mask"] = _pack(_reach(_dev(_parents(case))))
        if own:
            from paper_2609_26638_amd import dvs
            st["workspace"] = dvs.Workspace(dvs.tree_workspace_bytes(
                S, R, Hq, Hkv, D, table.shape[1], st["q"].dtype))
    return st


def _prepare_commit(case, seed, st, lens, table, need, stack, top, pool):
    S, R = case["S"], case["rows"]
    g = np.random.default_rng([seed, 5])
    parent = _parents(case)
    tokens = g.integers(0, 65536, (S, R))
    argmax = g.integers(0, 65536, (S, R))
    for s, path in enumerate(_paths(case, parent)):
        for a, b in zip([0] + path, path):
            argmax[s, a] = tokens[s, b]
    fields = dict(kv_len=lens, page_table=table, num_pages=need, free_stack=stack,
                  boundary=tokens[:, 0], draft=g.integers(0, 65536, (S, 15)),
                  out_tokens=g.integers(0, 65536, (S, MAX_NEW)),
                  out_count=g.integers(0, MAX_NEW, S), finished=_done(case))
    st.update(parent=_dev(parent), tokens=_dev(tokens), argmax=_dev(argmax))
    if own:
        from paper_2609_26638_amd import dvs, synth
        host = synth.PagedState(free_top=top, pool_pages=pool, max_pages=table.shape[1],
                                **{f: np.asarray(a, np.int32) for f, a in fields.items()})
        st["state"], st["before"] = dvs.DeviceState(host), dvs.DeviceState(host)
        st["handle"] = dvs.KVPools(*(list(p.unbind(0)) for p in st["pools"]))
        st["workspace"] = dvs.Workspace(dvs.accept_tree_workspace_bytes(S, R))
    else:
        fields = {f: _dev(a) for f, a in fields.items()}
        fields["free_top"] = _dev([top])
        st["state"], st["before"] = fields, {f: a.clone() for f, a in fields.items()}
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return RUN[state["case"]["kind"]](state)


def _run_masks(st):
    if own:
        from paper_2609_26638_amd import dvs
        return dvs.tree_masks(st["parent"])
    reach = _reach(st["parent"])
    return _pack(reach), (reach.sum(-1) - 1).to(torch.int32)


def _reach(parent):
    """[S, R, R]: row i has row j as itself or an ancestor.  A row of the
    padding, or below one, has none."""
    R = parent.shape[1]
    r = torch.arange(R, device=parent.device)
    edge = (parent.unsqueeze(-1) == r).float()
    reach = edge + torch.eye(R, device=parent.device)
    for _ in range(max(1, (R - 1).bit_length())):
        reach = ((reach @ reach) > 0).float()
    no = (parent < -1) | (parent >= r)
    return (reach > 0) & ((reach @ no.float().unsqueeze(-1)) == 0)


def _pack(reach):
    """Bit j % 32 of word j / 32."""
    S, R, _ = reach.shape
    W = (R + 31) // 32
    bits = torch.zeros((S, R, W * 32), dtype=torch.int64, device=reach.device)
    bits[..., :R] = reach
    words = (bits.view(S, R, W, 32) << torch.arange(32, device=reach.device)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _unpack(mask, R):
    bits = (mask.unsqueeze(-1) >> torch.arange(32, device=mask.device, dtype=torch.int32)) & 1
    return bits.flatten(-2)[..., :R].bool()


def _run_append(st):
    c = st["case"]
    if own:
        from paper_2609_26638_amd import dvs
        q = dvs.kv_append_rope(st["q"], st["k"], st["v"], *st["pools"], st["table"], st["kv_len"],
                               depth=st["depth"], theta=THETA, rot_dim=c["rot_dim"])
        return [q] + st["pools"]
    R = c["rows"]
    r = torch.arange(R, device="cuda")
    slot = st["kv_len"].long().unsqueeze(1) + r
    depth = r if st["depth"] is None else st["depth"].long()
    pos = (st["kv_len"].long().unsqueeze(1) + depth).double()
    half = c["rot_dim"] // 2
    i = torch.arange(half, device="cuda", dtype=torch.float64)
    angle = pos.unsqueeze(-1) * THETA ** (-i / max(half, 1))
    cs, sn = (f(angle).float().unsqueeze(2) for f in (torch.cos, torch.sin))

    def rotated(x):
        a, b, rest = x.float().split([half, half, x.shape[-1] - 2 * half], dim=-1)
        return torch.cat([a * cs - b * sn, b * cs + a * sn, rest], dim=-1).to(x.dtype)

    page = st["table"].gather(1, slot // PAGE).long()
    k_pool, v_pool = st["pools"]
    k_pool[page, :, slot % PAGE] = rotated(st["k"])
    v_pool[page, :, :, slot % PAGE] = st["v"]
    return [rotated(st["q"])] + st["pools"]


def _run_attn(st):
    c = st["case"]
    scale = c["head_dim"] ** -0.5
    if own:
        from paper_2609_26638_amd import dvs
        return dvs.attn_tree(st["q"], *st["pools"], st["table"], st["kv_len"], st["mask"], scale,
                             workspace=st["workspace"])
    S, R, Hq, Hkv, D = c["S"], c["rows"], c["heads"], c["kv_heads"], c["head_dim"]
    table = st["table"].long().clamp(min=0)
    k = st["pools"][0][table].float().permute(0, 2, 1, 3, 4).reshape(S, Hkv, -1, D)
    v = st["pools"][1][table].float().permute(0, 2, 1, 4, 3).reshape(S, Hkv, -1, D)
    key = torch.arange(k.shape[2], device="cuda")
    L = st["kv_len"].long().unsqueeze(1)
    tree = torch.zeros((S, R, k.shape[2]), dtype=torch.bool, device="cuda")
    tree.scatter_(2, (L + torch.arange(R, device="cuda")).unsqueeze(1).expand(S, R, R),
                  _unpack(st["mask"], R))
    seen = (key < L).unsqueeze(1) & (st["mask"] != 0).any(-1, keepdim=True) | tree
    q = st["q"].float().view(S, R, Hkv, Hq // Hkv, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, -1, D)
    z = (q @ k.transpose(-1, -2)).view(S, Hkv, Hq // Hkv, R, -1) * scale
    z = z.masked_fill(~seen[:, None, None], -math.inf)
    w = (z - z.amax(-1, keepdim=True).clamp(min=-1e30)).exp()
    total = w.sum(-1, keepdim=True)
    o = (w.view(S, Hkv, -1, k.shape[2]) @ v).view(S, Hkv, -1, R, D) / total.clamp(min=1e-30)
    return o.permute(0, 3, 1, 2, 4).reshape(S, R, Hq, D).to(st["q"].dtype)


FIELDS = ("kv_len", "page_table", "num_pages", "free_stack", "boundary", "draft", "out_tokens",
          "out_count", "finished", "free_top")


def _run_commit(st):
    c = st["case"]
    if own:
        from paper_2609_26638_amd import dvs
        st["state"].copy_from(st["before"])
        took, path = dvs.accept_commit_tree(st["state"], st["handle"], st["parent"], st["tokens"],
                                            st["argmax"], workspace=st["workspace"])
        return [took, path] + st["pools"] + [getattr(st["state"], f) for f in FIELDS]
    f, R = st["state"], c["rows"]
    for name in f:
        f[name].copy_(st["before"][name])
    parent, r = st["parent"].long(), torch.arange(R, device="cuda")
    live = f["finished"] == 0
    # the child that continues a row: the lowest whose token the row predicts
    up = parent.clamp(min=0)
    fits = (parent >= 0) & (st["tokens"] == st["argmax"].gather(1, up))
    follows = torch.full_like(parent, R).scatter_reduce(
        1, up, torch.where(fits, r, R), "amin", include_self=True)
    taken = fits & (follows.gather(1, up) == r) | (r == 0)
    reach = _reach(st["parent"])
    on = reach.any(-1) & ((reach.float() @ (~taken).float().unsqueeze(-1)).squeeze(-1) == 0)
    on = on & live.unsqueeze(1)
    depth = torch.where(on, reach.sum(-1) - 1, R)
    path = torch.full((c["S"], R + 1), -1, dtype=torch.int64, device="cuda")
    path.scatter_(1, depth, r.expand_as(depth))
    path = path[:, :R]
    path[~on[:, 0]] = -1
    A = (on.sum(-1) - 1).clamp(min=0)
    # tokens kept: the verifier's at every row of the path, while there is room
    k = torch.where(live, torch.minimum(A + 1, MAX_NEW - f["out_count"].long()), 0)
    kept = r < k.unsqueeze(1)
    tokens = st["argmax"].gather(1, path.clamp(min=0))
    s_of, i_of = kept.nonzero(as_tuple=True)
    f["out_tokens"][s_of, f["out_count"].long()[s_of] + i_of] = tokens[kept]
    f["boundary"].copy_(torch.where(
        k > 0, tokens.gather(1, (k - 1).clamp(min=0).unsqueeze(1)).squeeze(1), f["boundary"]))
    # cache rows of the path move to its front
    L, table = f["kv_len"].long(), f["page_table"].long()
    a, b = L[s_of] + path[kept], L[s_of] + i_of
    pa, pb = table[s_of, a // PAGE], table[s_of, b // PAGE]
    k_pool, v_pool = st["pools"]
    k_pool[:, pb, :, b % PAGE] = k_pool[:, pa, :, a % PAGE]
    v_pool[:, pb, :, :, b % PAGE] = v_pool[:, pa, :, :, a % PAGE]
    f["kv_len"] += k.to(torch.int32)
    f["out_count"] += k.to(torch.int32)
    f["finished"].copy_((~live | (f["out_count"] >= MAX_NEW)).to(torch.int32))
    # pages: surplus ones onto the stack, missing ones from its top
    n = f["num_pages"].long()
    need = (L + k + R + PAGE - 1) // PAGE
    j = torch.arange(table.shape[1], device="cuda")
    surplus = (j >= need.unsqueeze(1)) & (j < n.unsqueeze(1))
    missing = (j >= n.unsqueeze(1)) & (j < need.unsqueeze(1))
    back = f["page_table"].flip(1)[surplus.flip(1)]
    at = f["free_top"] + torch.arange(back.shape[0], device="cuda")
    f["free_stack"][at] = back
    f["page_table"][surplus] = -1
    at = f["free_top"] + back.shape[0] - missing.flatten().cumsum(0).view_as(missing)
    at = at[missing]
    f["page_table"][missing] = f["free_stack"][at]
    f["free_stack"][at] = -1
    f["free_top"] += back.shape[0] - at.shape[0]
    f["num_pages"].copy_(need)
    return [A.to(torch.int32), path.to(torch.int32)] + st["pools"] + [f[x] for x in FIELDS]


RUN = dict(masks=_run_masks, append=_run_append, attn=_run_attn, commit=_run_commit)


# ---------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return dict(masks=_exact_masks, append=_exact_append, attn=_exact_attn,
                commit=_exact_commit)[case["kind"]](st)


def _exact_masks(st):
    parent = st["parent"].cpu().numpy()
    S, R = parent.shape
    seen = np.zeros((S, R, (R + 31) // 32 * 32), np.uint8)
    depth = np.full((S, R), -1, np.int32)
    for r in range(R):
        p = parent[:, r]
        for s in range(S):
            if p[s] == -1 or (0 <= p[s] < r and depth[s, p[s]] >= 0):
                if p[s] >= 0:
                    seen[s, r] = seen[s, p[s]]
                    depth[s, r] = depth[s, p[s]]
                depth[s, r] += 1
                seen[s, r, r] = 1
    return np.packbits(seen, axis=-1, bitorder="little").view("<u4").view(np.int32), depth


def _exact_append(st):
    """A sequence at a time; pairs of elements as complex numbers."""
    c = st["case"]
    R, half = c["rows"], c["rot_dim"] // 2
    lens, table = st["kv_len"].cpu().numpy(), st["table"].cpu().numpy()
    k_pool, v_pool = (p.double() for p in st["pools"])
    freq = torch.from_numpy(THETA ** (-2.0 * np.arange(half) / max(2 * half, 1))).cuda()
    q_out = st["q"].double().clone()

    def turned(x, pos):
        z = torch.complex(x[..., :half], x[..., half:2 * half])
        z = z * torch.polar(torch.ones_like(freq), pos[:, None] * freq)[:, None]
        return torch.cat([z.real, z.imag, x[..., 2 * half:]], dim=-1)

    for s in range(c["S"]):
        d = torch.arange(R, device="cuda") if st["depth"] is None else st["depth"][s]
        pos = (int(lens[s]) + d.long()).double()
        q_out[s] = turned(st["q"][s].double(), pos)
        k = turned(st["k"][s].double(), pos)
        for j in range(lens[s] // PAGE, (lens[s] + R - 1) // PAGE + 1):
            a, b = max(j * PAGE, int(lens[s])), min((j + 1) * PAGE, int(lens[s]) + R)
            rows, slots = slice(a - int(lens[s]), b - int(lens[s])), slice(a - j * PAGE, b - j * PAGE)
            k_pool[table[s, j], :, slots] = k[rows].transpose(0, 1)
            v_pool[table[s, j], :, :, slots] = st["v"][s, rows].double().permute(1, 2, 0)
    return [q_out, k_pool, v_pool]


def _exact_attn(st):
    """A sequence and a KV head at a time, the keys gathered in order."""
    c = st["case"]
    R, G, D = c["rows"], c["heads"] // c["kv_heads"], c["head_dim"]
    lens, table = st["kv_len"].cpu().numpy(), st["table"].cpu().numpy()
    words = st["mask"].cpu().numpy().view(np.uint32)
    bits = np.unpackbits(words.view(np.uint8), axis=-1, bitorder="little")[..., :R].astype(bool)
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for s in range(c["S"]):
        L = int(lens[s])
        T = L + R
        pages = torch.from_numpy(table[s, :-(-T // PAGE)].astype(np.int64)).cuda()
        seen = np.concatenate([np.broadcast_to(bits[s].any(-1, keepdims=True), (R, L)), bits[s]], 1)
        seen = torch.from_numpy(np.repeat(seen, G, axis=0)).cuda()
        for h in range(c["kv_heads"]):
            k = st["pools"][0][pages, h].double().flatten(0, 1)[:T]
            v = st["pools"][1][pages, h].double().transpose(1, 2).flatten(0, 1)[:T]
            q = st["q"][s, :, h * G:(h + 1) * G].double().reshape(R * G, D)
            z = torch.where(seen, torch.mm(q, k.t()) / math.sqrt(D), -math.inf)
            w = torch.where(seen, torch.softmax(z, -1), 0.0)
            out[s, :, h * G:(h + 1) * G] = torch.mm(w, v).view(R, G, D)
    return out


def _exact_commit(st):
    """A sequence at a time, a row at a time."""
    c = st["case"]
    f = {k: v.cpu().numpy().copy() for k, v in st["state"].items()}
    parent, tokens, argmax = (st[n].cpu().numpy() for n in ("parent", "tokens", "argmax"))
    S, R = parent.shape
    took, paths = np.zeros(S, np.int32), np.full((S, R), -1, np.int32)
    table, stack, top = f["page_table"], f["free_stack"], int(f["free_top"][0])
    need, n, copies = np.zeros(S, np.int64), f["num_pages"].copy(), []
    for s in range(S):
        L = int(f["kv_len"][s])
        if not f["finished"][s]:
            path = [0]
            while True:
                fit = [r for r in range(R) if parent[s, r] == path[-1] >= 0
                       and tokens[s, r] == argmax[s, path[-1]]]
                if not fit:
                    break
                path.append(fit[0])
            took[s], paths[s, :len(path)] = len(path) - 1, path
            for i, row in enumerate(path):
                if f["out_count"][s] >= MAX_NEW:
                    break
                f["out_tokens"][s, f["out_count"][s]] = f["boundary"][s] = argmax[s, row]
                f["out_count"][s] += 1
                f["kv_len"][s] += 1
                if row != i:
                    copies.append(tuple((int(table[s, (L + x) // PAGE]), (L + x) % PAGE)
                                        for x in (row, i)))
            f["finished"][s] = int(f["out_count"][s] >= MAX_NEW)
        need[s] = -(-(int(f["kv_len"][s]) + R) // PAGE)
        for j in range(n[s] - 1, need[s] - 1, -1):
            stack[top], table[s, j] = table[s, j], -1
            top += 1
    for s in range(S):
        for j in range(n[s], need[s]):
            top -= 1
            table[s, j], stack[top] = stack[top], -1
    f["num_pages"][:], f["free_top"][0] = need, top
    pools = [p.clone() for p in st["pools"]]
    for (pa, a), (pb, b) in copies:
        pools[0][:, pb, :, b] = st["pools"][0][:, pa, :, a]
        pools[1][:, pb, :, :, b] = st["pools"][1][:, pa, :, :, a]
    return [took, paths] + pools + [f[x] for x in FIELDS]
