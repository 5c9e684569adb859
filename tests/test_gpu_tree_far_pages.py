"""GPU: the tree step on pages whose elements lie past 2^31 and whose bytes lie past 2^32 of the
pools: the same bits as on the pages of a small pool."""
import math

import numpy as np
import pytest
import torch

from oracle import tree as ot
from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import dev, i32, zero_err
from tests.test_gpu_tree_commit import drafted
from tests.test_oracle_pages import make_state
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu

PAGES, HKV, D = 600_000, 2, 128      # 2.46e9 elements, 4.9e9 bytes of bf16 a pool


@pytest.fixture(scope="module")
def pools():
    return [torch.empty((PAGES, HKV) + s, dtype=torch.bfloat16, device="cuda")
            for s in ((16, D), (D, 16))]


@pytest.mark.parametrize("columns", [0, 700])
@pytest.mark.parametrize("R,Hq", [(1, 4), (20, 4), (70, 16)])
def test_attention_and_append(pools, R, Hq, columns):
    lens = [300, 37, 5]
    rng = np.random.default_rng(R)
    st, k, v = cache(R, lens, R, HKV, D, "bf16")
    n = st.pool_pages
    small = [dev(k, "bf16"), dev(v, "bf16")]
    for big, s in zip(pools, small):
        big[PAGES - n:] = s
    far = [p[PAGES - n:] for p in pools]
    table = np.pad(st.page_table, ((0, 0), (0, max(0, columns - st.page_table.shape[1]))))
    kv_len, far_table = i32(st.kv_len), i32(table + (PAGES - n))
    table = i32(table)
    parent = random_parents(rng, 3, R)
    mask, depth = dvs.tree_masks(i32(parent))
    new = [dev(rounded(rng.standard_normal((3, R, h, D)), "bf16"), "bf16") for h in (Hq, HKV, HKV)]
    err = zero_err()
    got = []
    for p, t in ((small, table), (pools, far_table)):
        q = dvs.kv_append_rope(*new, *p, t, kv_len, depth=depth, err=err)
        got.append((q, dvs.attn_tree(q, *p, t, kv_len, mask, 1 / math.sqrt(D), err=err)))
    assert int(err) == 0
    # (padded rows of the rotated queries are left as they were: here, anything)
    assert torch.equal(got[0][0][depth >= 0], got[1][0][depth >= 0])
    assert torch.equal(got[0][1], got[1][1])
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(small, far))
    assert float(got[0][1].abs().max()) > 0


@pytest.mark.parametrize("R", [20, 70])
def test_commit(pools, R):
    """(up to 64 rows are accepted in the commit's launch)"""
    lens = [40, 9, 15]
    rng = np.random.default_rng(R)
    st, _, _ = make_state(R, lens, R)
    st.out_count[:] = 0
    n = st.pool_pages
    small = [torch.randint(-30000, 30000, (n, HKV) + s, dtype=torch.int16, device="cuda")
             for s in ((16, D), (D, 16))]
    for big, s in zip(pools, small):
        big[PAGES - n:] = s.view(torch.bfloat16)
    far = [p[PAGES - n:].view(torch.int16) for p in pools]
    parent = random_parents(rng, 3, R, padding=False)
    words = [i32(a) for a in (parent, *drafted(rng, parent))]
    near = dvs.DeviceState(st)
    up = lambda a: np.where(a >= 0, a + (PAGES - n), a)   # noqa: E731
    st.page_table = up(st.page_table)
    free = np.full(PAGES, -1, np.int32)
    free[:n] = up(st.free_stack)
    st.free_stack, st.pool_pages = free, PAGES
    away = dvs.DeviceState(st)
    out = [dvs.accept_commit_tree(s, dvs.KVPools([a.view(torch.bfloat16)], [b.view(torch.bfloat16)]), *words)
           for s, (a, b) in ((near, small), (away, pools))]
    assert int(near.err) == int(away.err) == 0
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert int(out[0][0].sum()) > 0 and torch.equal(near.kv_len, away.kv_len)
    assert all(torch.equal(a, b) for a, b in zip(small, far))
    held = near.page_table >= 0
    assert torch.equal(near.page_table[held] + (PAGES - n), away.page_table[held])
