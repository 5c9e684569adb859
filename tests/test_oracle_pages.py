"""Pins for the oracle's page calls (oracle/pages.py): what every sequence
sees in the cache, conservation of pages and counts, and a hand example."""
import numpy as np
import pytest

from oracle import pages as op
from paper_2609_26638_amd import synth


def make_state(seed, lens, window, max_new=20, draft=7, extra=40):
    """Pages for kv_len + window of every slot, scattered; pools [page, 16]
    whose entries are (page, slot) marks."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    st = synth.make_paged_state(rng, lens, window, int(lens.max() + window) // 16 + 4, True,
                                extra_pages=extra, n_causal=draft + 1, max_new=max_new)
    S = lens.size
    st.boundary[:] = rng.integers(0, 99, S)
    st.draft[:] = rng.integers(0, 99, st.draft.shape)
    st.out_tokens[:] = rng.integers(0, 99, st.out_tokens.shape)
    st.out_count[:] = rng.integers(0, max_new, S)
    pools = [rng.standard_normal((st.pool_pages, 16))]
    return st, np.zeros(st.pool_pages, np.int32), pools


def cache(st, pools, s):
    """What sequence s sees: its committed positions in order."""
    L = int(st.kv_len[s])
    return [np.concatenate([a[p] for p in st.page_table[s, :-(-L // 16)]])[:L] if L else a[:0, 0]
            for a in pools]


def check_counts(st, refs):
    """Holders by the tables equal refs + 1; free and held make up the pool."""
    held = np.zeros(st.pool_pages, np.int64)
    for s in range(st.kv_len.shape[0]):
        assert np.all(st.page_table[s, st.num_pages[s]:] == -1)
        for p in st.page_table[s, :st.num_pages[s]]:
            held[p] += 1
    free = st.free_stack[:st.free_top]
    assert np.all(st.free_stack[st.free_top:] == -1)
    held[free] += 1
    np.testing.assert_array_equal(held, refs + 1)
    assert not np.any(refs[free])


@pytest.mark.parametrize("share", [True, False])
def test_forks_see_what_their_source_sees(share):
    st, refs, pools = make_state(1, [33, 0, 16, 5, 40, 1], 9)
    before = [cache(st, pools, s) for s in range(6)]
    src, dst = [0, 2, 0, 1], [4, 3, 5, 1]
    assert op.kv_fork(st.copy(), refs.copy(), pools, src, dst, 9, share) == op.ERR_BAD_SLOT
    src, dst = [0, 2, 0], [4, 3, 5]
    assert op.kv_fork(st, refs, pools, src, dst, 9, share) == 0
    check_counts(st, refs)
    assert int(refs.sum()) == ((2 + 1 + 2) if share else 0)
    for a, b in zip(src, dst):
        for x, y in zip(cache(st, pools, b), before[a]):
            np.testing.assert_array_equal(x, y)
        for f in op.FIELDS:
            np.testing.assert_array_equal(getattr(st, f)[b], getattr(st, f)[a])
        assert st.num_pages[b] == -(-(st.kv_len[b] + 9) // 16)
        # the window's pages are nobody else's
        first = int(st.kv_len[b]) // 16
        assert not np.any(refs[st.page_table[b, first:st.num_pages[b]]])
    # written past its length, a fork leaves the others alone
    p = st.page_table[4, st.kv_len[4] // 16]
    pools[0][p, st.kv_len[4] % 16:] = 7.0
    for x, y in zip(cache(st, pools, 0) + cache(st, pools, 5), before[0] + before[0]):
        np.testing.assert_array_equal(x, y)


def test_hand_example():
    """Two slots of 17 and 0 positions, window 1: pages [2, 0] and [3], free
    1 (below) and 4 (top).  Forking 0 into 1 gives back 3, shares 2, pops 3."""
    st, refs, pools = make_state(2, [17, 0], 1, extra=0)
    st.pool_pages = 5
    st.page_table[:] = -1
    st.page_table[0, :2], st.page_table[1, 0] = [2, 0], 3
    st.free_stack = np.array([1, 4, -1, -1, -1], np.int32)
    st.free_top = 2
    refs = np.zeros(5, np.int32)
    pools = [np.arange(5.0)[:, None] * np.ones(16)]
    assert op.kv_fork(st, refs, pools, [0], [1], 1) == 0
    assert list(st.page_table[1, :3]) == [2, 3, -1] and list(refs) == [0, 0, 1, 0, 0]
    assert list(st.free_stack) == [1, 4, -1, -1, -1]
    assert pools[0][3, 0] == 0.0
    assert op.kv_release(st, refs, [0], 1) == 0     # 0 is freed, 2 is still held by slot 1
    assert list(st.page_table[0, :2]) == [0, -1] and list(refs) == [0] * 5
    assert list(st.page_table[1, :2]) == [2, 3]
    assert op.kv_compact(st, refs, pools) == (0, 1)
    assert list(st.page_table[1, :2]) == [2, 1] and list(st.free_stack) == [4, 3, -1, -1, -1]


def test_errors_leave_everything():
    st, refs, pools = make_state(3, [100, 3, 3], 4, extra=0)
    st0, p0 = st.copy(), pools[0].copy()
    st.free_top = 0
    assert op.kv_fork(st, refs, pools, [0], [1], 4, False) == op.ERR_POOL_EXHAUSTED
    assert op.kv_fork(st, refs, pools, [0], [1], 4000) == op.ERR_MAX_PAGES
    assert op.kv_fork(st, refs, pools, [0, 0], [1, 1], 4) == op.ERR_BAD_SLOT
    assert op.kv_fork(st, refs, pools, [0, 1], [1, 2], 4) == op.ERR_BAD_SLOT
    assert op.kv_release(st, refs, [3], 4) == op.ERR_BAD_SLOT
    assert op.kv_compact(st, refs, pools) == (op.ERR_BAD_PAGE, 0) or st0.free_top == 0
    for f in ("page_table", "num_pages", "free_stack", "kv_len"):
        np.testing.assert_array_equal(getattr(st, f), getattr(st0, f))
    np.testing.assert_array_equal(pools[0], p0)


def test_random_life_of_a_pool():
    """Forks, releases and compactions in turn keep counts, conservation and
    every untouched sequence's view."""
    rng = np.random.default_rng(9)
    S = 7
    st, refs, pools = make_state(9, [50, 0, 31, 32, 7, 90, 16], 6, extra=200)
    for step in range(60):
        seen = {s: cache(st, pools, s) for s in range(S)}
        kind = rng.integers(0, 3)
        if kind == 0:
            n = int(rng.integers(1, S))
            perm = rng.permutation(S)
            dst, src = perm[:n], rng.choice(perm[n:], n)
            assert op.kv_fork(st, refs, pools, src, dst, 6, bool(rng.integers(0, 2))) == 0
            for a, b in zip(src, dst):
                seen[b] = seen[a]
        elif kind == 1:
            gone = rng.permutation(S)[:int(rng.integers(1, 3))]
            if len(gone) < np.sum(st.kv_len > 0):
                assert op.kv_release(st, refs, gone, 6) == 0
                for b in gone:
                    seen[b] = [a[:0, 0] for a in pools]
        else:
            assert op.kv_compact(st, refs, pools)[0] == 0
            used = st.pool_pages - st.free_top
            assert all(p < used for s in range(S) for p in st.page_table[s, :st.num_pages[s]])
        check_counts(st, refs)
        for s in range(S):
            for x, y in zip(cache(st, pools, s), seen[s]):
                np.testing.assert_array_equal(x, y)
