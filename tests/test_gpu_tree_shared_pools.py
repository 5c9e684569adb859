"""GPU: accept_commit_tree on layers that share a cache, whose slots move once."""
import pytest

from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_commit_pages import LENS, both, every_other

pytestmark = pytest.mark.gpu


# (more than 64 layers: more than one launch takes)
@pytest.mark.parametrize("R", [40, 300])
@pytest.mark.parametrize("shares", [[0, 0], [0, 1, 0, 1], [1, 0, 0, 1, 1] + [0, 1] * 40],
                         ids=lambda s: f"{len(s)}layers")
def test_shared_caches_move_once(R, shares):
    b = both(R, max_new=2 * R, extra=200)
    k, v = b.handle.keep
    b.handle = dvs.KVPools([k[i] for i in shares], [v[i] for i in shares])
    if 1 not in shares:
        b.pools, b.bits = b.pools[:2], b.bits[:2]
    b.commit(*every_other(R))
    assert b.st.kv_len.tolist() == [n + (R + 1) // 2 for n in LENS]
