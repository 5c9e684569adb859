"""Trees and caches for the tests of the tree step."""
import numpy as np

from paper_2609_26638_amd import synth


def random_parents(rng, S, R, padding=True):
    """Random trees: runs, branches, other roots, shorter trees and holes."""
    p = np.where(rng.random((S, R)) < 0.6, np.arange(R) - 1,
                 (rng.random((S, R)) * np.arange(R)).astype(int))
    p[rng.random((S, R)) < 0.03] = -1
    p[:, 0] = -1
    if padding:
        p[rng.random((S, R)) < 0.04] = -2
        p[:, 0] = -1
        for s in range(S):
            if rng.random() < 0.5:
                p[s, rng.integers(1, R + 1):] = -7
    return p.astype(np.int32)


def cache(seed, lens, R, Hkv, D, dtype, spread=1.0, tail=None):
    """(state, K pool, V pool): float32 values that `dtype` holds exactly.  tail: what
    every slot past a sequence's window, and every free page, holds."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens)
    st = synth.make_paged_state(rng, lens, R, int(-(-(lens.max() + 2 * R) // 16)) + 2, True,
                                extra_pages=len(lens) * 4 + 4, max_new=64)
    k = rounded(spread * rng.standard_normal((st.pool_pages, Hkv, 16, D)), dtype)
    v = rounded(rng.standard_normal((st.pool_pages, Hkv, D, 16)), dtype)
    if tail is not None:
        kt, vt = np.full_like(k, tail), np.full_like(v, tail)
        for s, L in enumerate(lens):
            for t in range(L + R):
                pg = st.page_table[s, t // 16]
                kt[pg, :, t % 16], vt[pg, :, :, t % 16] = k[pg, :, t % 16], v[pg, :, :, t % 16]
        k, v = kt, vt
    return st, k, v


def rounded(a, dtype):
    a = np.asarray(a, np.float32)
    return synth.bf16_to_f32(synth.f32_to_bf16_bits(a)) if dtype == "bf16" else a
