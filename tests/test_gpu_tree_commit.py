"""GPU: accept_commit_tree against the oracle (oracle/tree.py): whole numbers and moved bits, so
the whole state and the pools have to be equal."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import i32
from tests.test_oracle_pages import make_state
from tests.tree_util import random_parents

pytestmark = pytest.mark.gpu


class Both:
    """One cache on the host (oracle) and on the device."""

    def __init__(self, seed, lens, R, layers=2, heads=2, D=64, dtype="bf16", **kw):
        self.st, _, _ = make_state(seed, lens, R, **kw)
        self.st.out_count[:] = 0
        rng = np.random.default_rng(seed + 1)
        it = np.int16 if dtype == "bf16" else np.int32
        P = self.st.pool_pages
        draw = lambda *s: rng.integers(-30000, 30000, (P, heads) + s).astype(it)   # noqa: E731
        self.pools = [draw(16, D) if i % 2 == 0 else draw(D, 16) for i in range(2 * layers)]
        tt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.bits = [torch.from_numpy(a.copy()).cuda() for a in self.pools]
        t = [b.view(tt) for b in self.bits]
        self.handle = dvs.KVPools(t[0::2], t[1::2])
        self.dev = dvs.DeviceState(self.st)

    def commit(self, parent, tokens, argmax, err=0, eos=-1, **kw):
        want = ot.accept_commit(self.st, self.pools, parent, tokens, argmax, eos)
        got = dvs.accept_commit_tree(self.dev, self.handle, i32(parent), i32(tokens), i32(argmax),
                                     eos_id=eos, **kw)
        torch.cuda.synchronize()
        assert want[0] == int(self.dev.err) == err
        self.dev.err.zero_()
        self.same()
        np.testing.assert_array_equal(got[0].cpu().numpy(), want[1])
        np.testing.assert_array_equal(got[1].cpu().numpy(), want[2])
        return want

    def same(self):
        got = self.dev.to_host(self.st)
        for f in dvs.DeviceState.FIELDS:
            np.testing.assert_array_equal(getattr(got, f), getattr(self.st, f), err_msg=f)
        assert got.free_top == self.st.free_top
        for i, (a, b) in enumerate(zip(self.bits, self.pools)):
            np.testing.assert_array_equal(a.cpu().numpy(), b, err_msg=f"pool {i}")


def drafted(rng, parent, vocab=3, follow=0.8):
    """Tokens and top-1s of which few values repeat (siblings that agree, ties for a parent) and
    most rows' top-1 is one of their children's tokens."""
    S, R = parent.shape
    tokens = rng.integers(0, vocab, (S, R))
    argmax = rng.integers(0, vocab, (S, R))
    for s in range(S):
        for r in range(R):
            kids = np.flatnonzero(parent[s] == r)
            if len(kids) and rng.random() < follow:
                argmax[s, r] = tokens[s, rng.choice(kids)]
    return tokens, argmax


CASES = [
    # lens, R, layers, heads, D, dtype
    ([0], 1, 1, 1, 64, "bf16"), ([15, 16, 17], 1, 2, 2, 96, "f32"), ([33, 0, 47, 5], 2, 1, 4, 128, "bf16"),
    ([7, 100, 31], 16, 2, 2, 64, "f32"), ([1, 12, 300], 17, 3, 1, 96, "bf16"),
    ([20, 63, 64, 65], 33, 2, 4, 64, "bf16"), ([5, 250], 64, 1, 8, 128, "f32"),
    ([40, 9], 65, 2, 2, 96, "bf16"), ([3], 200, 1, 2, 64, "bf16"), ([10, 0], 1024, 1, 1, 64, "f32"),
    (list(range(40, 110)), 5, 1, 1, 64, "bf16"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"S{len(c[0])}R{c[1]}l{c[2]}h{c[3]}D{c[4]}{c[5]}")
@pytest.mark.parametrize("deep", [False, True])
def test_rounds(case, deep):
    lens, R, layers, heads, D, dtype = case
    S = len(lens)
    rng = np.random.default_rng(R)
    b = Both(R, lens, R, layers, heads, D, dtype, max_new=3 * R + 9, extra=4 * S * (R // 16 + 2))
    for step in range(4):
        if deep:
            parent = np.tile(np.arange(-1, R - 1), (S, 1)).astype(np.int32)
            parent[:, 1::5] = -2 if step == 1 else 0
            parent[:, 0] = -1
        else:
            parent = random_parents(rng, S, R)
        if step == 2 and S > 1:
            parent[rng.integers(S), 0] = -2            # sits this step out
        if step == 3 and S > 1:
            s = rng.integers(S)
            b.st.finished[s] = 1
            b.dev.finished[s] = 1
        if (b.st.kv_len + 2 * R).max() > b.st.max_pages * 16:
            break
        b.commit(parent, *drafted(rng, parent), eos=1 if step == 1 else -1)


def test_lowest_child_padding_and_rows_that_are_no_trees():
    """Among children with the predicted token the lowest; a row that names itself or a later
    row is nobody's child."""
    parent = np.array([[-1, 2, 1, 0, 0, 3, 6, 5, 4]], np.int32)
    tokens = np.array([[0, 8, 8, 8, 8, 8, 8, 8, 8]])
    b = Both(1, [20], 9)
    want = b.commit(parent, tokens, np.full((1, 9), 8))
    assert want[2][0, :4].tolist() == [0, 3, 5, 7]


def test_budget_and_stop_token():
    parent = np.tile(np.array([-1, 0, 0, 1, 2, 2, 4], np.int32), (4, 1))
    tokens = np.tile([9, 5, 7, 8, 3, 3, 6], (4, 1))
    argmax = np.tile([7, 8, 3, 0, 6, 1, 2], (4, 1))
    b = Both(2, [30, 3, 14, 0], 7, max_new=20)
    for f in (b.st.out_count, b.dev.out_count):
        f[0], f[1], f[2] = 18, 20, 17
    b.commit(parent, tokens, argmax)
    assert b.st.finished.tolist() == [1, 1, 1, 0]
    b = Both(2, [30, 3, 14, 0], 7, max_new=20)
    b.commit(parent, tokens, argmax, eos=3)
    assert b.st.kv_len.tolist() == [32, 5, 16, 2]


@pytest.mark.parametrize("why", ["pool", "table"])
def test_a_commit_that_cannot_be_served_changes_nothing(why):
    R = 20
    parent = np.tile(np.arange(-1, R - 1), (2, 1)).astype(np.int32)
    parent[:, 2:] = np.arange(0, R - 2)      # paths of every other row
    tokens = argmax = np.zeros((2, R), int)
    b = Both(3, [38, 11], R, extra=8)
    if why == "pool":
        for f in (b.st.free_stack, b.dev.free_stack):
            f[:] = -1
        b.st.free_top = 0
        b.dev.free_top.zero_()
    else:
        # held pages stay; the table ends with them
        b.st.max_pages = b.dev.max_pages = int(b.st.num_pages.max())
        b.st.page_table = np.ascontiguousarray(b.st.page_table[:, :b.st.max_pages])
        b.dev.page_table = i32(b.st.page_table)
    before = [t.clone() for t in b.bits]
    b.commit(parent, tokens, argmax, err=1 if why == "pool" else 2)
    assert b.st.kv_len.tolist() == [38, 11]
    assert all(torch.equal(x, y) for x, y in zip(before, b.bits))


def test_many_layers_and_given_outputs():
    """More layers than one launch takes; outputs, workspace and stream given."""
    R, S = 6, 3
    rng = np.random.default_rng(0)
    b = Both(5, [14, 15, 3], R, layers=70, heads=1)
    parent = random_parents(rng, S, R, padding=False)
    ws = dvs.Workspace(dvs.accept_tree_workspace_bytes(S, R))
    ws.buf.fill_(255)
    acc = torch.empty(S, dtype=torch.int32, device="cuda")
    path = torch.empty((S, R), dtype=torch.int32, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b.commit(parent, *drafted(rng, parent), accept_out=acc, path_out=path, workspace=ws, stream=st)


def test_forked_slots_commit_apart():
    """Two slots that share full pages: each moves its own window only."""
    R = 12
    rng = np.random.default_rng(8)
    b = Both(9, [37, 4], R, extra=30)
    dvs.kv_fork(b.dev, b.handle, i32([0]), i32([1]), R)
    torch.cuda.synchronize()
    b.st = b.dev.to_host(b.st)
    b.pools = [t.cpu().numpy().copy() for t in b.bits]
    assert np.array_equal(b.st.page_table[0, :2], b.st.page_table[1, :2])
    for _ in range(3):
        parent = random_parents(rng, 2, R)
        b.commit(parent, *drafted(rng, parent))
