"""GPU: accept_commit_tree on tables with page ids outside the pool, against the oracle: a move that
needs such a page keeps the whole commit from happening."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import i32
from tests.test_gpu_tree_commit import Both

pytestmark = pytest.mark.gpu

LENS = [30, 7, 45]


def every_other(R):
    """Trees whose path is row 0, 2, 4, ..., with tokens and top-1s of 0."""
    parent = np.tile(np.maximum(np.arange(R) - 2, -1), (len(LENS), 1)).astype(np.int32)
    parent[:, 1::2] = -2
    return parent, np.zeros((len(LENS), R), int), np.zeros((len(LENS), R), int)


def both(R, **kw):
    """(tables wide enough for a whole window to be kept)"""
    b = Both(R, LENS, R, **kw)
    b.st.page_table = np.pad(b.st.page_table, ((0, 0), (0, R // 16 + 2)), constant_values=-1)
    b.st.max_pages = b.dev.max_pages = b.st.page_table.shape[1]
    b.dev.page_table = i32(b.st.page_table)
    return b


def plant(b, s, page, what):
    what = b.st.pool_pages if what == "end" else what
    b.st.page_table[s, page] = what
    b.dev.page_table[s, page] = what


# up to 64 rows: acceptance in the commit's launch
@pytest.mark.parametrize("R", [20, 64, 65, 300])
@pytest.mark.parametrize("bad", [-1, -5, "end", 1 << 30])
@pytest.mark.parametrize("page", ["first", "last"])
def test_nothing_changes_where_a_move_needs_the_page(R, bad, page):
    b = both(R, max_new=2 * R, extra=200)
    # the path's second row moves from slot 32 to slot 31; its last one from the last page
    plant(b, 0, 1 if page == "first" else (30 + (R - 1) // 2 * 2) // 16, bad)
    before = [t.clone() for t in b.bits]
    for _ in range(2):
        want = b.commit(*every_other(R), err=dvs.ERR_BAD_PAGE)
        assert want[1].tolist() == [(R - 1) // 2] * 3
    assert b.st.kv_len.tolist() == LENS
    assert all(torch.equal(x, y) for x, y in zip(before, b.bits))
    # without an error word the commit is refused as well
    words = [i32(a) for a in every_other(R)]
    sd = dvs._state_desc(b.dev, -1)
    sd.err_word = None
    ws = torch.empty(dvs.accept_tree_workspace_bytes(3, R), dtype=torch.uint8, device="cuda")
    rc = dvs.lib().accept_commit_tree(sd, b.handle.layers, len(b.handle.layers), b.handle.n_kv_heads,
                                      b.handle.head_dim, b.handle.dtype, R, *(w.data_ptr() for w in words),
                                      None, None, ws.data_ptr(), ws.numel(), dvs._stream())
    assert rc == 0
    torch.cuda.synchronize()
    b.same()


@pytest.mark.parametrize("R", [40, 64, 65, 300])
@pytest.mark.parametrize("why", ["budget", "stop token", "chain", "sits out", "finished"])
def test_a_page_that_no_move_needs(R, why):
    parent, tokens, argmax = every_other(R)
    b = both(R, max_new=8 if why == "budget" else 2 * R, extra=200)
    eos = -1
    last = (30 + R - 1) // 16
    if why == "stop token":
        eos, argmax[0, 14], tokens[0, 16] = 5, 5, 5
    elif why == "chain":
        parent[:] = np.arange(-1, R - 1)
    elif why == "sits out":
        parent[0, 0] = -2
    elif why == "finished":
        b.st.finished[0] = 1
        b.dev.finished[0] = 1
    plant(b, 0, last, -1)
    b.commit(parent, tokens, argmax, eos=eos)
    grown = {"budget": 8, "stop token": 8, "chain": R}.get(why, 0)
    assert int(b.st.kv_len[0]) == 30 + grown and int(b.st.kv_len[1]) > 7


@pytest.mark.parametrize("R", [20, 100])
def test_with_other_errors(R):
    b = both(R, max_new=2 * R, extra=8)
    for f in (b.st.free_stack, b.dev.free_stack):
        f[:] = -1
    b.st.free_top = 0
    b.dev.free_top.zero_()
    plant(b, 2, 3, -1)
    b.commit(*every_other(R), err=dvs.ERR_BAD_PAGE | dvs.ERR_POOL_EXHAUSTED)
