"""Oracle: a step over a tree of drafted tokens (float64, a row at a time).

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

A window's row 0 is the last committed token, row r continues row
``parent[s, r] < r`` (-1: attached to the cache alone; below -1, its own row or
a later one: padding).  Row r sees the cache and its ancestors, sits at slot
L + r and is rotated at position L + depth.
"""
from __future__ import annotations

import numpy as np

from . import decode

ERR_BAD_PAGE = 8
ERR_BAD_TREE = 64
PAGE = 16


def masks(parent: np.ndarray):
    """(visible [S, R, R] bool, depth [S, R], error word)."""
    S, R = parent.shape
    vis, depth, err = np.zeros((S, R, R), bool), np.full((S, R), -1, np.int32), 0
    for s in range(S):
        for r in range(R):
            p = int(parent[s, r])
            if p >= r:
                err |= ERR_BAD_TREE
                continue
            if p < -1 or (p >= 0 and depth[s, p] < 0):
                continue
            if p >= 0:
                vis[s, r] = vis[s, p]
            vis[s, r, r] = True
            depth[s, r] = int(depth[s, p]) + 1 if p >= 0 else 0
    return vis, depth, err


def words(vis: np.ndarray) -> np.ndarray:
    """Bit j % 32 of word j / 32, as int32."""
    S, R, _ = vis.shape
    out = np.zeros((S, R, -(-R // 32)), np.uint32)
    for j in range(R):
        out[:, :, j // 32] |= vis[:, :, j].astype(np.uint32) << np.uint32(j % 32)
    return out.view(np.int32)


def rotate(x: np.ndarray, pos: int, theta: float, rot_dim: int) -> np.ndarray:
    """x [heads, D] turned at one position."""
    h = rot_dim // 2
    out = np.array(x, np.float64)
    for i in range(h):
        a = pos * theta ** (-i / h)
        z = (out[:, i] + 1j * out[:, i + h]) * complex(np.cos(a), np.sin(a))
        out[:, i], out[:, i + h] = z.real, z.imag
    return out


def append_rope(q, k_new, v_new, k_pool, v_pool, table, kv_len, depth, theta, rot_dim):
    """Rotated queries; the pools (float64) are updated.  depth None: rows in order."""
    S, R = k_new.shape[:2]
    out = np.array(q, np.float64)
    for s in range(S):
        L = int(kv_len[s])
        for r in range(R):
            d = r if depth is None else int(depth[s, r])
            if d < 0:
                continue
            page, slot = int(table[s, (L + r) // PAGE]), (L + r) % PAGE
            out[s, r] = rotate(q[s, r], L + d, theta, rot_dim)
            k_pool[page, :, slot] = rotate(k_new[s, r], L + d, theta, rot_dim)
            v_pool[page, :, :, slot] = v_new[s, r]
    return out


def attention(q, k_pool, v_pool, table, kv_len, vis, scale):
    """(out, sum_k w_k |v_k|): the second bounds what an error of the weights does."""
    S, R, Hq, D = q.shape
    G = Hq // k_pool.shape[1]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for s in range(S):
        L = int(kv_len[s])
        for r in range(R):
            if not vis[s, r].any():
                continue
            keys = list(range(L)) + [L + j for j in range(R) if vis[s, r, j]]
            pages = table[s, [k // PAGE for k in keys]]
            slots = [k % PAGE for k in keys]
            for h in range(Hq):
                k = k_pool[pages, h // G, slots].astype(np.float64)
                v = v_pool[pages, h // G, :, slots].astype(np.float64)
                z = scale * (k @ q[s, r, h])
                w = np.exp(z - z.max())
                w /= w.sum()
                out[s, r, h], size[s, r, h] = w @ v, w @ np.abs(v)
    return out, size


def accepted(parent, tokens, argmax):
    """The rows of one sequence's accepted path, row 0 first."""
    path = [0]
    while True:
        for r in range(path[-1] + 1, len(parent)):
            if parent[r] == path[-1] and tokens[r] == argmax[path[-1]]:
                path.append(r)
                break
        else:
            return path


def kept(st, s, run, eos_id):
    """How many tokens of a run the budget and the stop token leave."""
    n = min(len(run), max(0, st.out_tokens.shape[1] - int(st.out_count[s])))
    return run.index(eos_id) + 1 if eos_id >= 0 and eos_id in run[:n] else n


def accept_commit(st, pools, parent, tokens, argmax, eos_id=-1):
    """Returns (error word, accepted [S], path [S, R]).  pools: K pools at even,
    V pools at odd places.  With an error, a slot to be moved whose page or whose
    target's is outside the pool among them, nothing is changed."""
    S, R = parent.shape
    took, path = np.zeros(S, np.int32), np.full((S, R), -1, np.int32)
    runs, idle = [[] for _ in range(S)], []
    for s in range(S):
        if st.finished[s] or parent[s, 0] != -1:
            idle.append(s)
            continue
        p = accepted(parent[s], tokens[s], argmax[s])
        took[s], path[s, :len(p)] = len(p) - 1, p
        runs[s] = [int(argmax[s, r]) for r in p]
    before, table, fin = st.kv_len.copy(), st.page_table.copy(), st.finished.copy()
    bad = 0
    for s in set(range(S)) - set(idle):
        moves = [(i, int(path[s, i])) for i in range(kept(st, s, runs[s], eos_id)) if path[s, i] != i]
        pages = [(int(before[s]) + t) // PAGE for m in moves for t in m]
        ids = [int(table[s, g]) for g in pages if 0 <= g < st.max_pages]
        if any(not 0 <= x < st.pool_pages for x in ids):
            bad = ERR_BAD_PAGE
    if bad:
        return bad | decode.kv_commit(st.copy(), took, argmax, R, 0, eos_id, block_runs=runs), took, path
    err = decode.kv_commit(st, took, argmax, R, 0, eos_id, block_runs=runs)
    if err:
        return err, took, path
    st.finished[idle] = fin[idle]
    for s in range(S):
        L = int(before[s])
        for i in range(int(st.kv_len[s]) - L):
            a, b = L + int(path[s, i]), L + i
            if a == b:
                continue
            pa, pb = table[s, a // PAGE], table[s, b // PAGE]
            for n, x in enumerate(pools):
                if n % 2 == 0:
                    x[pb, :, b % PAGE] = x[pa, :, a % PAGE]
                else:
                    x[pb, :, :, b % PAGE] = x[pa, :, :, a % PAGE]
    return 0, took, path
