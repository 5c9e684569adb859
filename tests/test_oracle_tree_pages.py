"""Pins for the oracle's tree commit on tables with page ids outside the pool."""
import numpy as np
import pytest

from oracle import tree as ot
from tests.test_oracle_pages import make_state

R = 20
PARENT = np.array([[-1, -2] + list(range(0, R - 2))] * 2, np.int32)     # path 0, 2, 4, ...
PARENT[:, 3::2] = -2


def state(max_new=64):
    st, _, _ = make_state(4, [30, 7], R, max_new=max_new)     # windows: pages 1 .. 3, 0 .. 1
    st.out_count[:] = 0
    pools = [np.arange(st.pool_pages * 16.0).reshape(st.pool_pages, 1, 16, 1).copy(),
             np.arange(st.pool_pages * 16.0).reshape(st.pool_pages, 1, 1, 16).copy()]
    return st, pools


def commit(st, pools, tokens=None, argmax=None, parent=PARENT, eos=-1):
    z = np.zeros((2, R), int)
    return ot.accept_commit(st, pools, parent, z if tokens is None else tokens,
                            z if argmax is None else argmax, eos)


@pytest.mark.parametrize("page", [1, 2, 3])
@pytest.mark.parametrize("bad", [-1, -5, "end", 1 << 30])
def test_a_page_that_a_move_needs(page, bad):
    st, pools = state()
    st.page_table[0, page] = st.pool_pages if bad == "end" else bad
    was, cache = st.copy(), [x.copy() for x in pools]
    err, took, path = commit(st, pools)
    # row 1 of the path (row 2) moves from slot 32 to 31: page 1 is a target, 2 and 3 sources
    assert err == ot.ERR_BAD_PAGE and took.tolist() == [9, 9] and path[0, :3].tolist() == [0, 2, 4]
    for f in ("kv_len", "page_table", "num_pages", "free_stack", "boundary", "out_tokens", "out_count",
              "finished"):
        np.testing.assert_array_equal(getattr(st, f), getattr(was, f))
    assert st.free_top == was.free_top and all(np.array_equal(a, b) for a, b in zip(pools, cache))


def test_a_page_that_no_move_needs():
    # truncated before the last page's rows are reached
    for kw in (dict(max_new=8), dict(eos=5)):
        st, pools = state(kw.get("max_new", 64))
        st.page_table[0, 3] = -1
        argmax, tokens = np.zeros((2, R), int), np.zeros((2, R), int)
        if "eos" in kw:
            argmax[0, 14], tokens[0, 16] = 5, 5
        assert commit(st, pools, tokens, argmax, eos=kw.get("eos", -1))[0] == 0
        assert st.kv_len.tolist() == ([38, 15] if "max_new" in kw else [38, 17])
    # a chain's slots stay where they are; one that sits out or has ended has no path
    st, pools = state()
    st.page_table[0, 2] = -1
    chain = np.tile(np.arange(-1, R - 1), (2, 1))
    assert commit(st, pools, parent=chain)[0] == 0
    for idle in (True, False):
        st, pools = state()
        st.page_table[0, 2] = -1
        parent = PARENT.copy()
        if idle:
            parent[0, 0] = -2
        else:
            st.finished[0] = 1
        assert commit(st, pools, parent=parent)[0] == 0
        assert st.kv_len.tolist() == [30, 17]
