"""GPU: commits of sequences whose lengths no table holds: DVS_ERR_MAX_PAGES (and, for the pages that
they would need, DVS_ERR_POOL_EXHAUSTED), and nothing changes."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import i32
from tests.test_gpu_tree_commit import Both

pytestmark = pytest.mark.gpu

S = 20


def tree(b, R):
    z = np.zeros((S, R), np.int32)
    parent = np.tile(np.arange(-1, R - 1), (S, 1))
    dvs.accept_commit_tree(b.dev, b.handle, i32(parent), i32(z), i32(z))


def chain(b, R):
    dvs.kv_commit(b.dev, i32(np.zeros(S)), i32(np.zeros((S, R))), R, 0)


def chain_with_acceptance(b, R):
    dvs.accept_commit(b.dev, i32(np.zeros((S, R))), R, 0)


@pytest.mark.parametrize("commit,R", [(tree, 7), (tree, 70), (chain, 7), (chain_with_acceptance, 7)])
@pytest.mark.parametrize("many", [False, True])
def test_lengths_near_two_to_the_31(commit, R, many):
    b = Both(1, [9 + s for s in range(S)], R, layers=1, heads=1, max_new=200)
    far = [2 ** 31 - 1 - 3 * s for s in range(S)]
    for s in range(S) if many else (4, 11):
        b.st.kv_len[s] = far[s]
    b.dev.kv_len.copy_(i32(b.st.kv_len))
    before = [t.clone() for t in b.bits]
    commit(b, R)
    torch.cuda.synchronize()
    assert int(b.dev.err) & dvs.ERR_MAX_PAGES
    b.same()
    assert all(torch.equal(x, y) for x, y in zip(before, b.bits))
