"""Sizes whose positions or page counts would pass 31 bits, refused on the host (nothing is
launched)."""
import ctypes

import pytest

from paper_2609_26638_amd import dvs
from tests.test_tree_refusals import _append, _attn, _commit, _state, needs_lib

WIDEST = 2 ** 27 - 4


@needs_lib
@pytest.mark.parametrize("R", [2 ** 31 - 1, 2 ** 31 - 10, 2 ** 31 - 16, 2 ** 28])
def test_append_of_windows_whose_pages_pass_31_bits(R):
    assert _append(R=R, S=1) == -2


@needs_lib
def test_tables_wider_than_31_bits_of_positions():
    one = dict(S=1, R=1, Hq=1, Hkv=1)
    for n in (WIDEST + 1, 2 ** 27, 2 ** 31 - 1):
        assert _append(max_pages=n) == -2
        assert _attn(**one, max_pages=n) == -2
        assert dvs.tree_workspace_bytes(1, 1, 1, 1, 64, n) == 0
        st = _state(max_pages=n)
        assert _commit(st=ctypes.byref(st)) == -2
    # one page fewer is refused for its workspace only
    assert dvs.tree_workspace_bytes(1, 1, 1, 1, 64, WIDEST) > 0
    assert _attn(**one, max_pages=WIDEST, nbytes=16) == -4
    st = _state(max_pages=WIDEST)
    assert _commit(st=ctypes.byref(st), nbytes=16) == -4


@needs_lib
def test_moves_of_more_threads_than_a_launch_has():
    st = _state(S=1024)
    nbytes = dvs.accept_tree_workspace_bytes(1024, 4)
    # two layers: 1024 * 4 * heads tasks
    assert _commit(st=ctypes.byref(st), nbytes=nbytes, heads=1 << 14) == -2
    assert _commit(st=ctypes.byref(st), nbytes=nbytes, heads=2 ** 31 - 1) == -2
    assert _commit(st=ctypes.byref(st), nbytes=16, heads=(1 << 14) - 1) == -4
    # the largest product that is taken: 1 * 1 * (2^25 - 2) with one layer, 2^25 - 1 is not
    st = _state(S=1)
    assert _commit(st=ctypes.byref(st), nbytes=16, n=1, heads=2 ** 25 - 2) == -4
    assert _commit(st=ctypes.byref(st), nbytes=16, n=1, heads=2 ** 25 - 1) == -2
