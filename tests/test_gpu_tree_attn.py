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


def run(case, dtype, vis, words, spread=1.0, tail=np.nan, seed=0, columns=0, **kw):
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
    table = st.page_table
    if table.shape[1] < columns:   # entries behind a sequence's pages are not read
        table = np.pad(table, ((0, 0), (0, columns - table.shape[1])), constant_values=1 << 30)
    out = dvs.attn_tree(dev(q, dtype), dev(k, dtype), dev(v, dtype), i32(table),
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


# more query rows than a wave, a workgroup and a CU's two workgroups take, over several tiles, a
# share that ends inside an item, and tables from a few pages to many
@pytest.mark.parametrize("case", [
    ([1500, 90], 33, 4, 4, 64), ([2100, 31, 700], 40, 8, 2, 64), ([1030, 1029], 64, 8, 2, 128),
    ([900, 2000], 36, 16, 4, 96), ([640, 1300, 5], 70, 16, 4, 128), ([777], 130, 4, 2, 96),
    ([50, 1, 0], 140, 4, 1, 64), ([1999, 64], 65, 8, 2, 128), ([96], 300, 4, 2, 128),
    ([127, 128, 129], 40, 2, 1, 128)],
    ids=lambda c: f"L{c[0][0]}x{len(c[0])}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_many_rows(case):
    lens, R = case[:2]
    vis, _, _ = ot.masks(random_parents(np.random.default_rng(R), len(lens), R))
    run(case, "bf16", vis, i32(ot.words(vis)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [([40, 7], 9, 4, 2, 64), ([100, 31], 20, 4, 2, 128),
                                  ([70, 300], 30, 8, 2, 96), ([33], 40, 16, 2, 128)],
                         ids=lambda c: f"R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
@pytest.mark.parametrize("columns", [0, 1100, 4200])
def test_rows_that_see_what_is_not_finite_and_rows_that_do_not(case, columns, dtype):
    """A drafted token's infinite or NaN value reaches its own row and its descendants', in the
    elements that have it; the other rows' results stay the bits that they are without it."""
    lens, R, Hq, Hkv, D = case
    S = len(lens)
    rng = np.random.default_rng(R)
    parent = random_parents(rng, S, R)
    vis, _, _ = ot.masks(parent)
    st, k, v = cache(R, lens, R, Hkv, D, dtype)
    q = dev(rounded(rng.standard_normal((S, R, Hq, D)), dtype), dtype)
    bad = v.copy()
    planted = []
    for s, L in enumerate(lens):
        for what, r, hk, d in ((np.inf, R // 3, 0, 1), (-np.inf, R // 2, Hkv - 1, D - 1),
                               (np.nan, R - 1, 0, D // 2 + 3), (-np.inf, R // 3, 0, 5)):
            bad[st.page_table[s, (L + r) // 16], hk, d, (L + r) % 16] = what
            planted.append((s, r, hk, d, what))
    words, scale = dvs.tree_masks(i32(parent))[0], 1 / math.sqrt(D)
    table = np.pad(st.page_table, ((0, 0), (0, max(0, columns - st.page_table.shape[1]))))
    args = i32(table), i32(st.kv_len), words, scale
    want = to_f64(dvs.attn_tree(q, dev(k, dtype), dev(v, dtype), *args)).copy()
    got = to_f64(dvs.attn_tree(q, dev(k, dtype), dev(bad, dtype), *args))
    G = Hq // Hkv
    hit = np.zeros(want.shape, bool)
    for s, r, hk, d, what in planted:
        for row in np.flatnonzero(vis[s, :, r]):
            at = (s, row, slice(hk * G, hk * G + G), d)
            assert np.all(np.isnan(got[at]) if np.isnan(what) else got[at] == what), (at, what)
            hit[at] = True
    assert np.array_equal(got[~hit], want[~hit])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("columns", [0, 1100, 4200])
@pytest.mark.parametrize("R,Hq,D", [(14, 4, 64), (30, 8, 128)])
def test_padded_queries_may_hold_anything(R, Hq, D, columns, dtype):
    """The other rows' results are the same bits whatever padded rows hold; so are those of rows
    beside one whose scores are large."""
    rng = np.random.default_rng(R)
    lens = [500, 90]
    st, k, v = cache(R, lens, R, 2, D, dtype)
    parent = random_parents(rng, 2, R, padding=False)
    parent[:, R // 2::3] = -2
    parent[:, R - 1] = 0
    vis, _, _ = ot.masks(parent)
    table = np.pad(st.page_table, ((0, 0), (0, max(0, columns - st.page_table.shape[1]))))
    args = (dev(k, dtype), dev(v, dtype), i32(table), i32(st.kv_len), i32(ot.words(vis)), D ** -0.5)
    q = rounded(rng.standard_normal((2, R, Hq, D)), dtype)
    want = to_f64(dvs.attn_tree(dev(q, dtype), *args))
    for what in (np.nan, np.inf, 1e30):
        other = q.copy()
        other[~vis.any(-1)] = rounded(what, dtype)
        other[:, R - 1] = rounded(40 * q[:, R - 1], dtype)
        got = to_f64(dvs.attn_tree(dev(other, dtype), *args))
        assert np.all(got[~vis.any(-1)] == 0)
        np.testing.assert_array_equal(got[:, :R - 1], want[:, :R - 1])
        assert np.all(np.isfinite(got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("columns", [130, 300, 1100])
@pytest.mark.parametrize("case", CASES[2:], ids=lambda c: f"L{c[0][0]}x{len(c[0])}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
def test_wide_tables(case, columns, dtype):
    """A table of many more pages than the sequences have: items in parts, few or many shares."""
    lens, R = case[:2]
    vis, _, _ = ot.masks(random_parents(np.random.default_rng(R + columns), len(lens), R))
    run(case, dtype, vis, i32(ot.words(vis)), columns=columns)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(40, 1, 4, 2, 64), (70, 5, 8, 2, 128), (33, 9, 8, 2, 96),
                                  (64, 33, 4, 4, 64), (65, 40, 8, 2, 128), (48, 17, 8, 1, 96),
                                  (100, 33, 8, 4, 64), (90, 40, 6, 2, 96), (70, 40, 8, 2, 96)],
                         ids=lambda c: f"S{c[0]}R{c[1]}H{c[2]}-{c[3]}D{c[4]}")
@pytest.mark.parametrize("columns", [0, 300])
def test_ragged_batches(case, columns, dtype):
    """Many sequences of nothing to 400 tokens, whole items or parts of them to a workgroup."""
    S, R, *rest = case
    rng = np.random.default_rng(S)
    lens = [int(x) for x in rng.integers(0, 400, S)]
    lens[3] = lens[S - 1] = 0
    vis, _, _ = ot.masks(random_parents(rng, S, R))
    run((lens, R, *rest), dtype, vis, i32(ot.words(vis)), columns=columns)


def test_fp32_batches_that_give_every_wave_two_groups():
    rng = np.random.default_rng(2)
    lens = [int(x) for x in rng.integers(0, 2000, 12)]
    vis, _, _ = ot.masks(random_parents(rng, 12, 30))
    run((lens, 30, 8, 4, 128), "f32", vis, i32(ot.words(vis)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_wave_has_lanes(dtype):
    """The sequences' tiles are found in registers up to 64 of them, in LDS beyond."""
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 300, 70)]
    for R, Hq, Hkv in ((1, 4, 2), (40, 2, 2)):
        vis, _, _ = ot.masks(random_parents(rng, 70, R))
        run((lens, R, Hq, Hkv, 64), dtype, vis, i32(ot.words(vis)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_launch_takes(dtype):
    """1030 sequences of a token or none, whose calls go out in two launches."""
    lens = [i % 3 for i in range(1030)]
    vis = np.ones((1030, 1, 1), bool)
    vis[5::7] = False
    run((lens, 1, 2, 1, 64), dtype, vis, i32(ot.words(vis)))


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
