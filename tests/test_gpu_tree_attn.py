"""GPU: attn_tree against the oracle (oracle/tree.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.gpu_util import max_rel_err, to_f64
from tests.test_gpu_tree_append import dev, i32, zero_err
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu


def check(got, want, size, dtype):
    """bf16: every weight is rounded once (half a step, 2^-8 of it: together 2^-8 of size =
    sum w |v|), and the output once (2^-8 of it).  What is summed in 32 bits (scores of up to 128
    products, weights, outputs) adds under 2^-12 of size at scores below 32.
    fp32: 1e-5 of each output vector's largest element, the framework's bound."""
    if dtype == "bf16":
        tol = 2.0 ** -8 * (np.abs(want) + size) + 2.0 ** -12 * size + 1e-30
        worst = np.max(np.abs(got - want) / tol)
        assert worst <= 1, worst
    else:
        live = np.abs(want).max(-1) > 0
        assert np.all(got[~live] == 0)
        assert max_rel_err(got[live], want[live]) <= 1e-5


def run(case, dtype, vis, words, spread=1.0, tail=np.nan, seed=0, **kw):
    lens, R, Hq, Hkv, D = case
    st, k, v = cache(seed + R, lens, R, Hkv, D, dtype, spread=spread, tail=tail)
    rng = np.random.default_rng(seed)
    q = rounded(rng.standard_normal((len(lens), R, Hq, D)) * spread, dtype)
    # slots of rows that no row sees hold anything
    for s, L in enumerate(lens):
        for r in np.flatnonzero(~vis[s].any(0)):
            pg, sl = st.page_table[s, (L + r) // 16], (L + r) % 16
            k[pg, :, sl], v[pg, :, :, sl] = np.nan, np.inf
    scale = 1 / math.sqrt(D)
    want, size = ot.attention(q.astype(float), k, v, st.page_table, st.kv_len, vis, scale)
    err = zero_err()
    out = dvs.attn_tree(dev(q, dtype), dev(k, dtype), dev(v, dtype), i32(st.page_table),
                        i32(st.kv_len), words, scale, err=err, **kw)
    assert int(err) == 0
    got = to_f64(out)
    assert np.all(np.isfinite(got))
    assert np.all(got[~vis.any(-1)] == 0)
    check(got, want, size, dtype)
    return out


CASES = [
    # lens, R, Hq, Hkv, D
    ([0], 1, 4, 4, 64), ([1], 1, 4, 1, 96), ([15, 16, 17], 1, 16, 4, 128),
    ([63, 64, 65, 127, 128], 1, 8, 8, 64), ([300, 0, 700], 1, 32, 8, 64), ([1500], 1, 16, 1, 128),
    ([0, 5], 2, 8, 2, 64), ([33, 47], 7, 12, 2, 96), ([129, 1, 400], 8, 4, 4, 128),
    ([64, 250], 16, 4, 2, 64), ([500], 17, 16, 4, 96), ([31, 90], 32, 4, 1, 128),
    ([260, 3], 33, 8, 2, 64), ([700, 100], 37, 16, 4, 128), ([200, 64], 64, 8, 2, 96),
    ([50], 65, 16, 4, 64), ([111, 17], 100, 6, 2, 128), ([20], 257, 4, 1, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"L{c[0][0]}x{len(c[0])}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_trees(case, dtype):
    lens, R = case[:2]
    parent = random_parents(np.random.default_rng(R), len(lens), R)
    vis, _, _ = ot.masks(parent)
    run(case, dtype, vis, dvs.tree_masks(i32(parent))[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [CASES[i] for i in (0, 2, 5, 6, 9, 11, 13, 14, 17)],
                         ids=lambda c: f"L{c[0][0]}x{len(c[0])}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_no_mask_is_causal(case, dtype):
    lens, R = case[:2]
    vis = np.tile(np.tri(R, dtype=bool), (len(lens), 1, 1))
    a = run(case, dtype, vis, None)
    b = run(case, dtype, vis, i32(ot.words(vis)))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_mask(dtype):
    """Bits that no tree has: rows that see later rows, everything, or nothing; a row without
    itself; bits past the window are no slots."""
    S, R = 3, 45
    rng = np.random.default_rng(9)
    vis = rng.random((S, R, R)) < 0.3
    vis[0, 3], vis[0, 4], vis[1, :, 7], vis[2] = False, True, False, False
    vis[2, 5, 44] = True
    words = ot.words(vis)
    words[..., -1] |= np.int32(-1 << (R % 32))
    words[~vis.any(-1)] = 0
    run(([70, 0, 333], R, 8, 2, 64), dtype, vis, i32(words))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("spread", [0.01, 2.3])
def test_flat_and_peaked_scores(dtype, spread):
    """Nearly uniform weights, and scores that span tens (largest below 32 at 2.3 * 2.3)."""
    case = ([900, 40], 24, 8, 2, 64)
    vis, _, _ = ot.masks(random_parents(np.random.default_rng(1), 2, 24))
    run(case, dtype, vis, i32(ot.words(vis)), spread=spread)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R", [1, 9, 40])
def test_long_ragged_batch(dtype, R):
    """Long beside empty caches, more work items than the chip holds at once, and pages out of
    order."""
    lens = [3000, 0, 17, 1200, 64, 1, 2222]
    case = (lens, R, 8, 4, 64)
    vis, _, _ = ot.masks(random_parents(np.random.default_rng(R), len(lens), R))
    run(case, dtype, vis, i32(ot.words(vis)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_does_not_feel_the_batch_nor_the_workspace(dtype):
    """Rerun: the same bits, also with a workspace full of NaN and shared by another shape; a
    given output is written whole."""
    case = ([800, 3], 20, 8, 2, 96)
    vis, _, _ = ot.masks(random_parents(np.random.default_rng(2), 2, 20))
    words = i32(ot.words(vis))
    a = run(case, dtype, vis, words)
    ws = dvs.Workspace(64 << 20)
    ws.buf.fill_(255)
    out = torch.full_like(a, float("nan"))
    b = run(case, dtype, vis, words, workspace=ws, out=out)
    assert b is out and torch.equal(a, b)
    run(([5], 3, 4, 4, 64), dtype, np.tri(3, dtype=bool)[None], None, workspace=ws)
    assert torch.equal(run(case, dtype, vis, words, workspace=ws), a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_errors(dtype):
    S, R, Hq, Hkv, D = 4, 6, 4, 2, 64
    lens = [40, 300, 20, 9]
    vis = np.tile(np.tri(R, dtype=bool), (S, 1, 1))
    st, k, v = cache(3, lens, R, Hkv, D, dtype)
    q = rounded(np.random.default_rng(0).standard_normal((S, R, Hq, D)), dtype)
    want, size = ot.attention(q.astype(float), k, v, st.page_table, st.kv_len, vis, 0.125)
    pt, kv = st.page_table.copy(), st.kv_len.copy()
    pt[1, 5], pt[1, 6] = st.pool_pages, -5
    kv[2], kv[3] = st.max_pages * 16 - R + 1, -4
    err = zero_err()
    out = dev(np.full(q.shape, 7.0), dtype)
    dvs.attn_tree(dev(q, dtype), dev(k, dtype), dev(v, dtype), i32(pt), i32(kv), None, 0.125, err=err,
                  out=out)
    assert int(err) == dvs.ERR_BAD_PAGE | dvs.ERR_MAX_PAGES
    got = to_f64(out)
    assert np.all(got[2:] == 7.0)
    check(got[:1], want[:1], size[:1], dtype)
