"""Size queries return, whatever the sizes (sums of 32 bits may wrap, a division by
zero would end the process); vocabularies at the sampler's limit (no GPU needed)."""
import ctypes
import os
import random

import pytest

from paper_2609_26638_amd import dvs
from tests.test_chunk_keys_refusals import _model
from tests.test_filter_pages_refusals import _accept, _sample

pytestmark = pytest.mark.skipif(not os.path.exists(dvs.LIB_PATH),
                                reason="libdvs.so not built (run __graft_entry__.build())")
SIZES = [-1, 0, 1, 2, 7, 16, 33, 64, 1000, 1 << 16, 1 << 22, 1 << 29, 1 << 30, (1 << 31) - 1]


@pytest.mark.parametrize("dtype", [dvs.DVS_F32, dvs.DVS_BF16])
def test_any_sizes(dtype):
    L, r = dvs.lib(), random.Random(dtype)
    for _ in range(20000):
        S, B, P, pages = (r.choice(SIZES) for _ in range(4))
        chunk = r.choice([0, 64, 128, 16384])
        model = _model(dtype)
        model.n_kv_heads = r.choice([1, 4])
        model.n_heads, model.head_dim = model.n_kv_heads * r.choice([1, 4]), r.choice([64, 96, 128])
        m = ctypes.byref(model)
        L.dvs_attn_workspace_bytes(S, B, P, model.n_heads, model.n_kv_heads, model.head_dim, pages,
                                   chunk, dtype)
        L.dvs_step_workspace_bytes(m, S, B, P, pages, chunk)
        L.dvs_prefill_workspace_bytes(m, S, P, B, pages, chunk)
        L.dvs_diffusion_workspace_bytes(m, S, B, pages, chunk)
        L.dvs_sampled_round_workspace_bytes(m, S, B, pages, chunk)
        L.dvs_filtered_round_workspace_bytes(m, S, B, pages, chunk)
        L.dvs_accept_workspace_bytes(S, B, P)
        L.dvs_kv_workspace_bytes(S, pages)


def test_vocabularies_past_the_limit():
    L, V = dvs.lib(), (1 << 22) + 1
    assert _sample(L, V=V, ld=V) == -1 and b"2^22" in L.dvs_last_error()
    assert _accept(L, V=V, vld=V, dld=V) == -1 and b"2^22" in L.dvs_last_error()
    assert dvs.accept_workspace_bytes(2, 3, V) == 0 and dvs.accept_workspace_bytes(2, 3, V - 1) > 0
