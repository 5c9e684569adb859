"""GPU: tree_masks and kv_append_rope against the oracle (oracle/tree.py)."""
import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.gpu_util import to_f64
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu


def i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(
        torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def zero_err():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---- masks

@pytest.mark.parametrize("R", [1, 2, 5, 31, 32, 33, 63, 64, 65, 96, 97, 128, 129, 300, 640, 1000, 1024])
@pytest.mark.parametrize("S", [1, 6])
def test_masks(S, R):
    rng = np.random.default_rng(R * 10 + S)
    parent = random_parents(rng, S, R)
    vis, depth, _ = ot.masks(parent)
    err = zero_err()
    mask, got = dvs.tree_masks(i32(parent), err=err)
    np.testing.assert_array_equal(got.cpu().numpy(), depth)
    np.testing.assert_array_equal(mask.cpu().numpy(), ot.words(vis))
    assert int(err) == 0


@pytest.mark.parametrize("R", [64, 200, 1024])
def test_masks_of_chains_stars_and_rows_that_are_no_trees(R):
    r = np.arange(R)
    parent = np.stack([r - 1, np.where(r == 0, -1, 0), np.full(R, -1), np.full(R, -2),
                       np.where(r % 3 == 2, r, r - 1), np.where(r == R // 2, R + 5, r - 1),
                       np.where(r == 7, 2**31 - 1, np.where(r == 9, -2**31, r // 2 - (r == 0)))])
    vis, depth, bad = ot.masks(parent)
    err = zero_err()
    mask, got = dvs.tree_masks(i32(parent), err=err)
    np.testing.assert_array_equal(got.cpu().numpy(), depth)
    np.testing.assert_array_equal(mask.cpu().numpy(), ot.words(vis))
    assert int(err) == bad == ot.ERR_BAD_TREE
    assert int((mask != 0).any(-1).sum()) == int((depth >= 0).sum())
    dvs.tree_masks(i32(parent))            # no error word


# ---- append

def run_append(q, k, v, kp, vp, st, depth, theta, rot, dtype, **kw):
    pools = [dev(kp, dtype), dev(vp, dtype)]
    err = zero_err()
    out = dvs.kv_append_rope(q, k, v, *pools, i32(st.page_table), i32(st.kv_len),
                             depth=None if depth is None else i32(depth), theta=theta, rot_dim=rot,
                             err=err, **kw)
    torch.cuda.synchronize()
    return out, pools, int(err)


def bound(a, b, dtype):
    """How far a rotated element a' = a cos - b sin may be off: sines and cosines within
    2^-22.5 of themselves absolutely (the reduced angle's own rounding, 2^-26 of a quarter turn,
    and two half-steps), three roundings of 2^-24 in the products and their sum, then one to the
    type: half a step, 2^-8 of the value in bf16."""
    size = (np.abs(a) + np.abs(b)) * 2.0 ** -21
    return size + (2.0 ** -8 * (np.abs(a) + np.abs(b)) if dtype == "bf16" else 0)


def check_turned(got, want, src, rot, dtype):
    h = rot // 2
    np.testing.assert_array_equal(got[..., rot:], src[..., rot:])
    if not h:
        return
    a, b = src[..., :h], src[..., h:rot]
    tol = bound(a, b, dtype)
    if dtype == "bf16":      # half a step of what came out, not of both inputs' size
        tol = (np.abs(a) + np.abs(b)) * 2.0 ** -21 * (1 + 2.0 ** -8)
        for part in (slice(0, h), slice(h, rot)):
            assert np.all(np.abs(got[..., part] - want[..., part]) <= tol + 2.0 ** -8 * np.abs(want[..., part]))
    else:
        for part in (slice(0, h), slice(h, rot)):
            assert np.all(np.abs(got[..., part] - want[..., part]) <= tol)


CASES = [
    # lens, R, Hq, Hkv, D, rot, tree
    ([0], 1, 4, 4, 64, 64, False),
    ([15], 1, 4, 2, 96, 96, False),
    ([16, 31, 1], 1, 16, 4, 128, 128, False),
    ([15, 16, 17, 0], 2, 8, 2, 64, 32, True),
    ([3, 300], 16, 4, 1, 96, 48, True),
    ([16, 9], 17, 12, 2, 128, 16, True),
    ([5, 4096, 77], 37, 8, 2, 64, 0, True),
    ([100001, 7], 64, 4, 4, 96, 96, True),
    ([0, 13], 200, 2, 1, 64, 64, False),
    ([1, 2, 3, 4, 5, 6, 7, 8, 9], 5, 16, 1, 128, 112, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"L{c[0][0]}R{c[1]}H{c[2]}-{c[3]}D{c[4]}r{c[5]}")
@pytest.mark.parametrize("layout", ["fused", "odd"])
def test_append(case, dtype, layout):
    lens, R, Hq, Hkv, D, rot, tree = case
    S = len(lens)
    rng = np.random.default_rng(R + D)
    # what the call neither reads nor may change: NaN
    st, kp, vp = cache(R, lens, R, Hkv, D, dtype)
    kp[:], vp[:] = np.nan, np.nan
    parts = [rounded(rng.standard_normal((S, R, h, D)), dtype) for h in (Hq, Hkv, Hkv)]
    depth = ot.masks(random_parents(rng, S, R))[1] if tree else None
    if layout == "fused":        # the rows of one projection
        x = torch.cat([dev(p, dtype).flatten(2) for p in parts], -1)
        q, k, v = (t.unflatten(-1, (-1, D)) for t in x.split([Hq * D, Hkv * D, Hkv * D], -1))
    else:                        # rows that start on no 16 bytes, sequences apart
        def odd(p):
            h = p.shape[2] * D
            buf = torch.full((S, R + 1, h + 3), float("nan"), device="cuda",
                             dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
            t = buf[:, 1:, 1:1 + h]
            t.copy_(dev(p, dtype).flatten(2))
            return t.unflatten(-1, (-1, D))
        q, k, v = map(odd, parts)
    want_k, want_v = kp.astype(float), vp.astype(float)
    want = ot.append_rope(*parts, want_k, want_v, st.page_table, st.kv_len, depth, 10000.0, rot)
    filler = dev(np.full(parts[0].shape, 7.0), dtype)
    out, pools, err = run_append(q, k, v, kp, vp, st, depth, 10000.0, rot, dtype, q_out=filler)
    assert err == 0
    got = to_f64(out)
    live = np.ones((S, R), bool) if depth is None else depth >= 0
    assert np.all(got[~live] == 7.0)
    check_turned(got[live], want[live], parts[0][live].astype(float), rot, dtype)
    gk, gv = to_f64(pools[0]), to_f64(pools[1])
    np.testing.assert_array_equal(gv, want_v)                # copies, NaN elsewhere
    assert np.array_equal(np.isnan(gk), np.isnan(want_k))
    for s in range(S):
        for r in np.flatnonzero(live[s]):
            pg, sl = st.page_table[s, (lens[s] + r) // 16], (lens[s] + r) % 16
            check_turned(gk[pg, :, sl], want_k[pg, :, sl], parts[1][s, r].astype(float), rot, dtype)


def test_append_in_place_without_queries_and_other_bases():
    S, R, Hq, Hkv, D = 2, 19, 4, 2, 64
    rng = np.random.default_rng(0)
    st, kp, vp = cache(1, [40, 7], R, Hkv, D, "f32")
    parts = [rng.standard_normal((S, R, h, D)).astype(np.float32) for h in (Hq, Hkv, Hkv)]
    wk, wv = kp.astype(float), vp.astype(float)
    want = ot.append_rope(*parts, wk, wv, st.page_table, st.kv_len, None, 500000.0, D)
    q, k, v = (dev(p, "f32") for p in parts)
    out, pools, _ = run_append(q, k, v, kp, vp, st, None, 500000.0, None, "f32", q_out=q)
    assert out is q
    check_turned(to_f64(q), want, parts[0].astype(float), D, "f32")
    none, pools2, _ = run_append(None, k, v, kp, vp, st, None, 500000.0, None, "f32")
    assert none is None
    assert all(torch.equal(a, b) for a, b in zip(pools, pools2))
    with pytest.raises(dvs.DvsError, match="in place"):
        x = torch.zeros((S, R, 2 * Hq, D), device="cuda")[:, :, :Hq]
        dvs.kv_append_rope(x, k, v, *pools, i32(st.page_table), i32(st.kv_len),
                           q_out=torch.as_strided(x, (S, R, Hq, D), (R * Hq * D, Hq * D, D, 1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D,rot", [(4, 6, 64, 64), (1, 9, 96, 32), (24, 3, 128, 128)])
def test_append_of_a_large_batch_is_that_of_its_parts(Hq, Hkv, D, rot, dtype):
    """A workgroup takes the more heads of a page the more pages there are: the same bits."""
    S, R = 720, 33
    rng = np.random.default_rng(D)
    lens = rng.integers(0, 20, S)
    st, kp, vp = cache(D, lens, R, Hkv, D, dtype)
    parent = random_parents(rng, S, R)
    depth = i32(ot.masks(parent)[1])
    parts = [dev(rng.standard_normal((S, R, h, D)), dtype) for h in (Hq, Hkv, Hkv)]
    table, kv_len = i32(st.page_table), i32(st.kv_len)
    a, b = ([dev(kp, dtype), dev(vp, dtype)] for _ in range(2))
    kw = dict(rot_dim=rot)
    out = dvs.kv_append_rope(*parts, *a, table, kv_len, depth=depth, **kw, q_out=torch.zeros_like(parts[0]))
    for s in range(0, S, 40):
        c = slice(s, s + 40)
        got = dvs.kv_append_rope(*(p[c] for p in parts), *b, table[c], kv_len[c], depth=depth[c],
                                 **kw, q_out=torch.zeros_like(parts[0][c]))
        assert torch.equal(out[c], got)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    dvs.kv_append_rope(*parts, *b, table, kv_len, depth=depth, **kw, q_out=parts[0])
    live = depth >= 0
    assert torch.equal(parts[0][live], out[live])


def test_append_far_positions_keep_their_angle():
    """At position 16 million, where 32 bits no longer tell neighbouring angles apart, with the
    cache's own length short: the depth carries the distance."""
    S, R, D = 1, 4, 64
    rng = np.random.default_rng(3)
    st, kp, vp = cache(2, [9], R, 1, D, "f32")
    parts = [rng.standard_normal((S, R, 1, D)).astype(np.float32) for _ in range(3)]
    depth = np.array([[16_000_001, 16_777_217, 2_000_000_011, 123_456_789]])
    wk, wv = kp.astype(float), vp.astype(float)
    want = ot.append_rope(*parts, wk, wv, st.page_table, st.kv_len, depth, 10000.0, D)
    out, _, _ = run_append(*(dev(p, "f32") for p in parts), kp, vp, st, depth, 10000.0, D, "f32")
    # the angle itself, 2e9 quarter turns, is known to 2^-53 of itself on both sides: 4e-7
    a = np.abs(parts[0]).astype(float)
    tol = (a[..., :32] + a[..., 32:]) * (2.0 ** -21 + 2 * 2.1e9 * 2.0 ** -52)
    err = np.abs(to_f64(out) - want)
    assert np.all(err[..., :32] <= tol) and np.all(err[..., 32:] <= tol)


def test_append_reports_bad_pages_and_full_tables():
    S, R, Hq, Hkv, D = 3, 20, 4, 2, 64
    rng = np.random.default_rng(5)
    st, kp, vp = cache(4, [10, 30, 50], R, Hkv, D, "bf16")
    parts = [rounded(rng.standard_normal((S, R, h, D)), "bf16") for h in (Hq, Hkv, Hkv)]
    wk, wv = kp.astype(float), vp.astype(float)
    want = ot.append_rope(*parts, wk, wv, st.page_table, st.kv_len, None, 10000.0, D)
    page = int(st.page_table[1, 2])
    st.page_table[1, 2] = st.pool_pages                # slots 32 .. 47 of sequence 1
    st.kv_len[2] = st.max_pages * 16 - R + 1           # one row too many
    out, pools, err = run_append(*(dev(p, "bf16") for p in parts), kp, vp, st, None, 10000.0, D,
                                 "bf16", q_out=dev(np.full(parts[0].shape, 7.0), "bf16"))
    assert err == dvs.ERR_BAD_PAGE | dvs.ERR_MAX_PAGES
    got = to_f64(out)
    assert np.all(got[2] == 7.0)
    check_turned(got[:2], want[:2], parts[0][:2].astype(float), D, "bf16")
    wv[page] = vp[page]
    old = st.page_table[2]
    for t in range(50, 50 + R):
        pg = old[t // 16]
        wv[pg, :, :, t % 16] = vp[pg, :, :, t % 16]
    np.testing.assert_array_equal(to_f64(pools[1]), wv)
    np.testing.assert_array_equal(to_f64(pools[0])[page], kp[page])
    st.kv_len[:] = [-1, 2**31 - 3, 10]
    run = run_append(*(dev(p, "bf16") for p in parts), kp, vp, st, None, 10000.0, D, "bf16")
    assert run[2] & dvs.ERR_MAX_PAGES
