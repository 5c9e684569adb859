"""GPU: accept_commit_tree over batches whose trees several waves of the commit's launch accept, on
both sides of the sizes that it takes (64 sequences, 64 rows), against the oracle."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import i32
from tests.test_gpu_tree_commit import Both, drafted
from tests.tree_util import random_parents

pytestmark = pytest.mark.gpu


def widen(b, steps, R):
    """Room in the tables for whole windows kept."""
    b.st.page_table = np.pad(b.st.page_table, ((0, 0), (0, steps * R // 16 + 1)), constant_values=-1)
    b.st.max_pages = b.dev.max_pages = b.st.page_table.shape[1]
    b.dev.page_table = i32(b.st.page_table)


@pytest.mark.parametrize("R", [1, 2, 33, 64, 65])
@pytest.mark.parametrize("S", [5, 8, 31, 63, 64, 65])
def test_batches(S, R):
    """Random trees, chains and deep paths; some sequences have ended, some sit out, some meet the
    stop token, some the budget."""
    rng = np.random.default_rng(100 * S + R)
    lens = rng.integers(0, 90, S).tolist()
    b = Both(S + R, lens, R, layers=1, heads=2, max_new=2 * R + 7, extra=12 * S)
    widen(b, 3, R)
    count = rng.integers(0, R + 8, S)
    fin = rng.random(S) < 0.15
    for st in (b.st, b.dev):
        for i in range(S):
            st.out_count[i], st.finished[i] = int(count[i]), int(fin[i])
    for step in range(3):
        parent = random_parents(rng, S, R)
        deep = rng.random(S) < 0.5
        parent[deep] = np.maximum(np.arange(R) - rng.integers(1, 3), -1 if R == 1 else 0)
        parent[:, 0] = np.where(rng.random(S) < 0.1, -2, -1)
        took = b.commit(parent, *drafted(rng, parent, vocab=4), eos=3 if step == 1 else -1)[1]
        assert R == 1 or step or took.max() > 0


@pytest.mark.parametrize("S", [33, 64])
def test_each_sequence_keeps_a_run_of_its_own(S):
    """Path lengths and tokens that differ from sequence to sequence: 64 - s rows of the chain."""
    R = 64
    b = Both(S, [s % 20 for s in range(S)], R, layers=1, heads=1, max_new=R, extra=8 * S)
    widen(b, 1, R)
    for f in (b.st.finished, b.st.out_count):
        f[:] = 0
    b.dev.finished.zero_()
    b.dev.out_count.zero_()
    parent = np.tile(np.arange(-1, R - 1), (S, 1)).astype(np.int32)
    tokens = np.arange(S)[:, None] * 1000 + np.arange(R)[None]
    argmax = tokens + 1
    for s in range(S):
        argmax[s, R - 1 - s] = -7 - s
    want = b.commit(parent, tokens, argmax)
    assert want[1].tolist() == [R - 1 - s for s in range(S)]
    assert b.st.out_tokens[S - 1, :R - S + 1].tolist() == [1000 * (S - 1) + i + 1 for i in range(R - S)] + [-6 - S]


@pytest.mark.parametrize("S,R", [(3, 20), (64, 64), (3, 100), (1024, 9)])
def test_outputs_may_be_left_out(S, R):
    """NULL accept_out and path_out: the same state and cache, with a workspace of any contents."""
    rng = np.random.default_rng(R)
    b = Both(R, rng.integers(0, 60, S).tolist(), R, layers=2, heads=1, max_new=2 * R, extra=S * (R // 16 + 2))
    widen(b, 1, R)
    b.st.out_count[:] = 0
    b.dev.out_count.zero_()
    parent = random_parents(rng, S, R)
    tokens, argmax = drafted(rng, parent)
    want = ot.accept_commit(b.st, b.pools, parent, tokens, argmax)
    assert want[0] == 0 and want[1].max() > 0
    words = [i32(a) for a in (parent, tokens, argmax)]
    ws = torch.full((dvs.accept_tree_workspace_bytes(S, R),), 255, dtype=torch.uint8, device="cuda")
    rc = dvs.lib().accept_commit_tree(dvs._state_desc(b.dev, -1), b.handle.layers, len(b.handle.layers),
                                      b.handle.n_kv_heads, b.handle.head_dim, b.handle.dtype, R,
                                      *(w.data_ptr() for w in words), None, None, ws.data_ptr(), ws.numel(),
                                      dvs._stream())
    assert rc == 0
    torch.cuda.synchronize()
    assert int(b.dev.err) == 0
    b.same()


@pytest.mark.parametrize("R", [7, 64, 100, 1024])
def test_masks_without_depths(R):
    parent = i32(random_parents(np.random.default_rng(R), 5, R))
    want = dvs.tree_masks(parent)[0]
    mask = torch.full_like(want, -1)
    rc = dvs.lib().tree_masks(parent.data_ptr(), 5, R, mask.data_ptr(), None, None, dvs._stream())
    assert rc == 0
    assert torch.equal(mask, want)
