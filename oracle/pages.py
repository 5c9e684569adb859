"""Oracle: forking, releasing and compacting the pages of a paged cache.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__``).

``st`` is a synth.PagedState-like object, ``refs`` [pool] the holders of each
page beyond the first, ``pools`` a list of arrays whose first axis is the
page.  Every function works slot by slot and page by page, changes nothing
when it returns an error word, and returns 0 otherwise.
"""
from __future__ import annotations

import numpy as np

ERR_POOL_EXHAUSTED = 1
ERR_MAX_PAGES = 2
ERR_BAD_PAGE = 8
ERR_BAD_SLOT = 32
PAGE = 16

FIELDS = ("kv_len", "boundary", "draft", "out_tokens", "out_count", "finished")


def _ceil(n):
    return -(-int(n) // PAGE)


def _pages(st, s):
    return [int(p) for p in st.page_table[s, :st.num_pages[s]]]


def _assign(st, refs, pools, src, dst, window, share):
    S, pool = st.kv_len.shape[0], st.pool_pages
    err = 0
    for i, b in enumerate(dst):
        if not 0 <= b < S or b in list(dst[:i]):
            err |= ERR_BAD_SLOT
        if src is not None and (not 0 <= src[i] < S or b in list(src)):
            err |= ERR_BAD_SLOT
    if err:
        return err
    lens = [int(st.kv_len[a]) for a in src] if src is not None else [0] * len(dst)
    for L, b in zip(lens, dst):
        if _ceil(L + window) > st.max_pages:
            err |= ERR_MAX_PAGES
    for b in dst:
        if any(not 0 <= p < pool for p in _pages(st, b)):
            err |= ERR_BAD_PAGE
    if err:
        return err
    # what the destinations give back
    left = refs.copy()
    freed = []
    for b in dst:
        for p in _pages(st, b):
            left[p] -= 1
            if left[p] < 0:
                left[p] = 0
                freed.append(p)
    stack = [int(p) for p in st.free_stack[:st.free_top]] + sorted(freed, reverse=True)
    full = [L // PAGE if share else 0 for L in lens]
    if sum(_ceil(L + window) - f for L, f in zip(lens, full)) > len(stack):
        return ERR_POOL_EXHAUSTED
    refs[:] = left
    for i, b in enumerate(dst):
        L, row = lens[i], []
        for j in range(_ceil(L + window)):
            if j < full[i]:
                p = int(st.page_table[src[i], j])
                refs[p] += 1
            else:
                p = stack.pop()
                if j * PAGE < L:
                    for a in pools:
                        a[p] = a[st.page_table[src[i], j]]
            row.append(p)
        st.page_table[b] = -1
        st.page_table[b, :len(row)] = row
        st.num_pages[b] = len(row)
        if src is not None:
            for f in FIELDS:
                getattr(st, f)[b] = getattr(st, f)[src[i]]
        else:
            st.kv_len[b] = st.boundary[b] = st.out_count[b] = 0
            st.finished[b] = 1
    st.free_stack[:] = -1
    st.free_stack[:len(stack)] = stack
    st.free_top = len(stack)
    return 0


def kv_fork(st, refs, pools, src, dst, window, share=True):
    return _assign(st, refs, pools, list(src), list(dst), window, share)


def kv_release(st, refs, slots, window):
    return _assign(st, refs, [], None, list(slots), window, False)


def kv_compact(st, refs, pools):
    """Returns (error word, pages moved)."""
    S, pool = st.kv_len.shape[0], st.pool_pages
    held = sorted({p for s in range(S) for p in _pages(st, s)})
    free = sorted(int(p) for p in st.free_stack[:st.free_top])
    if sorted(held + free) != list(range(pool)):
        return ERR_BAD_PAGE, 0
    U = len(held)
    moves = dict(zip([p for p in held if p >= U], [p for p in free if p < U]))
    for a, b in moves.items():
        for x in pools:
            x[b] = x[a]
        refs[b], refs[a] = refs[a], 0
    for s in range(S):
        for j in range(st.num_pages[s]):
            p = int(st.page_table[s, j])
            st.page_table[s, j] = moves.get(p, p)
    st.free_stack[:] = -1
    st.free_stack[:pool - U] = np.arange(pool - 1, U - 1, -1)
    return 0, len(moves)
