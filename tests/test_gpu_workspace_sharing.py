"""GPU: one workspace for attn_hybrid_block and for calls that leave anything in it."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_gpu_tree_append import dev, i32
from tests.test_gpu_tree_commit import Both, drafted
from tests.tree_util import cache, random_parents, rounded

pytestmark = pytest.mark.gpu

S, N, HQ, HKV, D = 3, 5, 8, 2, 64


def test_attention_after_other_calls():
    """The same bits as with a workspace of its own, after every other call that takes one."""
    rng = np.random.default_rng(0)
    st, k, v = cache(1, [900, 40, 333], 40, HKV, D, "bf16")
    new = [dev(rounded(rng.standard_normal((S, 2 * N, h, D)), "bf16"), "bf16") for h in (HQ, HKV, HKV)]
    pools, table, kv_len = (dev(k, "bf16"), dev(v, "bf16")), i32(st.page_table), i32(st.kv_len)
    ws = dvs.Workspace(64 << 20)

    def attend(workspace):
        return dvs.attn_hybrid_block(*new, *pools, table, kv_len, N, N, 0.125, workspace=workspace)

    want = attend(None)
    assert torch.equal(attend(ws), want)
    parent = random_parents(rng, S, 40)
    q = dev(rng.standard_normal((S, 40, HQ, D)), "bf16")
    mask = dvs.tree_masks(i32(parent))[0]
    wide = i32(np.pad(st.page_table, ((0, 0), (0, 400))))
    b = Both(2, [20, 3, 31], 40, layers=1, heads=HKV, max_new=99, extra=40)
    z = torch.randn((S, 6, 100), device="cuda")
    draft, u = i32(rng.integers(0, 100, (S, 5))), torch.rand((S, 6), device="cuda")
    others = {
        "attn_tree": lambda: dvs.attn_tree(q, *pools, wide, kv_len, mask, 0.125, workspace=ws),
        "accept_commit_tree": lambda: b.commit(parent, *drafted(rng, parent), workspace=ws),
        "accept_sampled": lambda: dvs.accept_sampled(z, z[:, :5], draft, u, workspace=ws),
        "kv_compact": lambda: dvs.kv_compact(b.dev, b.handle, workspace=ws),
        "kv_release": lambda: dvs.kv_release(b.dev, i32([1]), 40, workspace=ws),
        "kv_fork": lambda: dvs.kv_fork(b.dev, b.handle, i32([0]), i32([1]), 40, workspace=ws),
    }
    for name, call in others.items():
        call()
        for _ in range(2):
            assert torch.equal(attend(ws), want), name
    assert int(b.dev.err) == 0
