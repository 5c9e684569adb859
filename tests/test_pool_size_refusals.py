"""Pools whose page counts would not fit the page calls' 32-bit sums are refused on
the host (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2609_26638_amd import dvs
from tests.test_filter_pages_refusals import F, N, _fork, _layers, _state

pytestmark = pytest.mark.skipif(not os.path.exists(dvs.LIB_PATH),
                                reason="libdvs.so not built (run __graft_entry__.build())")


@pytest.mark.parametrize("pages,rc", [((1 << 29) + 1, -1), ((1 << 31) - 1, -1), (1 << 29, -4)])
def test_page_calls(pages, rc):
    L, st, big = dvs.lib(), _state(num_pool_pages=pages), 1 << 20
    assert (dvs.kv_workspace_bytes(4, pages) > 0) == (rc == -4)
    assert _fork(L, st=st) == rc
    assert L.kv_release(ctypes.byref(st), F, 1, F, 4, F, big, N) == rc
    assert L.kv_compact(ctypes.byref(st), F, _layers(), 2, 2, 64, 1, N, F, big, N) == rc
