"""accept_commit_tree on layers that share half a cache (nothing is launched)."""
import pytest

from paper_2609_26638_amd import dvs
from tests.test_tree_refusals import _commit, needs_lib


@needs_lib
@pytest.mark.parametrize("layer", [dict(v_pool=0x2000), dict(k_pool=0x2000)])
def test_one_pool_of_a_pair_is_refused(layer):
    assert _commit(layer=layer) == -1
    assert b"share" in dvs.lib().dvs_last_error()
