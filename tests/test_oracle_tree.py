"""Pins for the oracle of the tree step (oracle/tree.py)."""
import numpy as np
import pytest

from oracle import attention as oa
from oracle import model as om
from oracle import tree as ot
from tests.tree_util import cache, random_parents


def test_hand_tree():
    #        0
    #      1   2        5: padding   6 below it   7: a root of its own   8: names a later row
    #    3       4
    vis, depth, err = ot.masks(np.array([[-1, 0, 0, 1, 2, -2, 5, -1, 9, 4]], np.int32))
    assert err == ot.ERR_BAD_TREE
    assert depth.tolist() == [[0, 1, 1, 2, 2, -1, -1, 0, -1, 3]]
    seen = [np.flatnonzero(v).tolist() for v in vis[0]]
    assert seen == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [], [], [7], [], [0, 2, 4, 9]]
    assert ot.words(vis)[0, :, 0].tolist() == [1, 3, 5, 11, 21, 0, 0, 128, 0, 1 + 4 + 16 + 512]


def test_chain_is_causal_and_words_pass_32():
    R = 40
    vis, depth, err = ot.masks(np.arange(-1, R - 1, dtype=np.int32)[None])
    assert err == 0 and np.array_equal(vis[0], np.tri(R, dtype=bool))
    assert depth[0].tolist() == list(range(R))
    w = ot.words(vis)
    assert w.shape == (1, R, 2) and w[0, 39].tolist() == [-1, 255] and w[0, 31, 0] == -1


def test_rotation_is_the_models():
    x = np.random.default_rng(0).standard_normal((3, 8))
    want = om.rope(x[None], np.array([37.0]), 10000.0)[0]
    np.testing.assert_allclose(ot.rotate(x, 37, 10000.0, 8), want, atol=1e-12)
    part = ot.rotate(x, 37, 10000.0, 4)
    np.testing.assert_array_equal(part[:, 4:], x[:, 4:])
    # scores go by the distance alone
    y = np.random.default_rng(1).standard_normal((3, 8))
    dots = [(ot.rotate(x, a, 500.0, 8) * ot.rotate(y, a - 5, 500.0, 8)).sum(-1) for a in (5, 905)]
    np.testing.assert_allclose(dots[0], dots[1], atol=1e-9)


def test_chain_attention_is_the_causal_window():
    rng = np.random.default_rng(2)
    S, R, Hq, Hkv, D = 2, 5, 4, 2, 8
    st, k, v = cache(3, [19, 0], R, Hkv, D, "f32")
    q = rng.standard_normal((S, R, Hq, D))
    kn, vn = rng.standard_normal((2, S, R, Hkv, D))
    want = oa.attn_hybrid_block(q, kn, vn, k.astype(float), v.astype(float), st.page_table,
                                st.kv_len, R, 0, 0.3)
    k, v = k.astype(float), v.astype(float)
    ot.append_rope(q, kn, vn, k, v, st.page_table, st.kv_len, None, 1e4, 0)
    vis, _, _ = ot.masks(np.tile(np.arange(-1, R - 1), (S, 1)).astype(np.int32))
    got, size = ot.attention(q, k, v, st.page_table, st.kv_len, vis, 0.3)
    np.testing.assert_allclose(got, want, atol=1e-12)
    assert np.all(size >= np.abs(got) - 1e-12)


@pytest.mark.parametrize("seed", range(4))
def test_a_row_of_a_tree_is_the_end_of_its_chain(seed):
    """A row's output equals that of its ancestors verified alone as a chain."""
    rng = np.random.default_rng(seed)
    R, Hq, Hkv, D = 12, 2, 1, 8
    parent = random_parents(rng, 1, R)
    vis, depth, _ = ot.masks(parent)
    st, k, v = cache(seed, [21], R, Hkv, D, "f32")
    q = rng.standard_normal((1, R, Hq, D))
    kn, vn = rng.standard_normal((2, 1, R, Hkv, D))
    k1, v1 = k.astype(float), v.astype(float)
    rq = ot.append_rope(q, kn, vn, k1, v1, st.page_table, st.kv_len, depth, 50.0, 8)
    got, _ = ot.attention(rq, k1, v1, st.page_table, st.kv_len, vis, 0.4)
    for r in range(R):
        rows = np.flatnonzero(vis[0, r])
        if not len(rows):
            assert not got[0, r].any()
            continue
        k2, v2 = k.astype(float), v.astype(float)
        cq = ot.append_rope(q[:, rows], kn[:, rows], vn[:, rows], k2, v2, st.page_table, st.kv_len,
                            None, 50.0, 8)
        chain = np.tri(len(rows), dtype=bool)[None]
        want, _ = ot.attention(cq, k2, v2, st.page_table, st.kv_len, chain, 0.4)
        np.testing.assert_allclose(got[0, r], want[0, -1], atol=1e-12)


def test_hand_acceptance():
    parent = [-1, 0, 0, 1, 2, 2, 4]
    tokens = [9, 5, 7, 8, 3, 3, 6]
    assert ot.accepted(parent, tokens, [7, 8, 3, 0, 6, 1, 2]) == [0, 2, 4, 6]
    assert ot.accepted(parent, tokens, [5, 1, 3, 0, 6, 1, 2]) == [0, 1]
    assert ot.accepted(parent, tokens, [1, 1, 3, 0, 6, 1, 2]) == [0]


def test_commit_keeps_the_path_and_its_slots():
    R = 7
    st, k, v = cache(5, [30, 3, 14], R, 1, 2, "f32")
    parent = np.array([[-1, 0, 0, 1, 2, 2, 4]] * 3, np.int32)
    parent[2, 0] = -2                                  # no tree this step
    tokens = np.array([[9, 5, 7, 8, 3, 3, 6]] * 3)
    argmax = np.array([[7, 8, 3, 0, 6, 1, 2]] * 3)
    st.finished[1] = 1
    before = st.copy()
    k0, v0 = k.copy(), v.copy()
    err, took, path = ot.accept_commit(st, [k, v], parent, tokens, argmax)
    assert err == 0 and took.tolist() == [3, 0, 0]
    assert path.tolist() == [[0, 2, 4, 6, -1, -1, -1], [-1] * 7, [-1] * 7]
    assert st.kv_len.tolist() == [34, 3, 14] and st.out_count.tolist() == [4, 0, 0]
    assert st.out_tokens[0, :4].tolist() == [7, 3, 6, 2] and st.boundary[0] == 2
    assert st.num_pages.tolist() == [-(-(n + R) // 16) for n in (34, 3, 14)]
    pt = before.page_table[0]
    for i, r in enumerate([0, 2, 4, 6]):
        a, b = 30 + r, 30 + i
        np.testing.assert_array_equal(k[pt[b // 16], :, b % 16], k0[pt[a // 16], :, a % 16])
        np.testing.assert_array_equal(v[pt[b // 16], :, :, b % 16], v0[pt[a // 16], :, :, a % 16])


def test_commit_stops_and_budget():
    R = 7
    parent = np.array([[-1, 0, 0, 1, 2, 2, 4]], np.int32)
    tokens, argmax = np.array([[9, 5, 7, 8, 3, 3, 6]]), np.array([[7, 8, 3, 0, 6, 1, 2]])
    st, k, v = cache(6, [5], R, 1, 2, "f32")
    assert ot.accept_commit(st, [k, v], parent, tokens, argmax, eos_id=3)[0] == 0
    assert st.kv_len[0] == 7 and st.finished[0] == 1 and st.boundary[0] == 3
    st, k, v = cache(6, [5], R, 1, 2, "f32")
    st.out_count[0] = 61                               # 64 in all
    assert ot.accept_commit(st, [k, v], parent, tokens, argmax)[0] == 0
    assert st.kv_len[0] == 8 and st.finished[0] == 1 and st.out_tokens[0, 61:].tolist() == [7, 3, 6]
