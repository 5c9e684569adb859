"""Every size query and model call refuses a chunk_keys that is no multiple of 64,
negative or too large, before anything is planned or launched (no GPU needed)."""
import ctypes
import os

import pytest

from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.skipif(not os.path.exists(dvs.LIB_PATH),
                                reason="libdvs.so not built (run __graft_entry__.build())")
F = ctypes.c_void_p(0x1000)     # never dereferenced: validation fails first
BAD = [1, 16, 63, 65, 100, -1, -64, 16448, 1 << 30]


def _model(dtype):
    layers = (dvs.DvsLayer * 1)()
    for n, _ in dvs.DvsLayer._fields_:
        setattr(layers[0], n, 0x1000)
    return dvs.DvsModel(dtype, 1, 1000, 64, 1, 1, 64, 64, 1e4, 1e-6, 0x1000, 0x1000, 0x1000, layers)


def _state():
    v = dict(S=4, max_pages=8, num_pool_pages=64, draft_width=2, max_new=16, eos_id=-1)
    v.update({n: 0x1000 for n, _ in dvs.DvsState._fields_[6:]})
    return dvs.DvsState(**v)


@pytest.mark.parametrize("dtype", [dvs.DVS_F32, dvs.DVS_BF16])
@pytest.mark.parametrize("chunk", BAD)
def test_size_queries(chunk, dtype):
    L, m = dvs.lib(), ctypes.byref(_model(dtype))
    for c, fits in ((chunk, False), (0, True), (64, True), (16384, True)):
        for got in (L.dvs_attn_workspace_bytes(4, 2, 2, 1, 1, 64, 8, c, dtype),
                    L.dvs_step_workspace_bytes(m, 4, 2, 2, 8, c),
                    L.dvs_prefill_workspace_bytes(m, 4, 9, 2, 8, c),
                    L.dvs_diffusion_workspace_bytes(m, 4, 2, 8, c),
                    L.dvs_sampled_round_workspace_bytes(m, 4, 2, 8, c),
                    L.dvs_filtered_round_workspace_bytes(m, 4, 2, 8, c)):
            assert (got > 0) == fits


@pytest.mark.parametrize("dtype", [dvs.DVS_F32, dvs.DVS_BF16])
@pytest.mark.parametrize("chunk", BAD)
def test_model_calls(chunk, dtype):
    L, N, big = dvs.lib(), None, 1 << 40
    m, st = ctypes.byref(_model(dtype)), ctypes.byref(_state())
    steps = ctypes.c_int32(0)
    for name, call in (
            ("draft_verify_step", lambda: L.draft_verify_step(m, st, 2, 2, chunk, N, N, N, F, big, N)),
            ("multidraft_step", lambda: L.multidraft_step(m, st, 2, chunk, N, N, N, F, big, N)),
            ("literal_round", lambda: L.literal_round(m, st, 2, chunk, N, N, N, F, big, N)),
            ("diffusion_denoise", lambda: L.diffusion_denoise(m, st, 2, 0.5, F, F, chunk, N, N, N, F, big, N)),
            ("diffusion_block", lambda: L.diffusion_block(m, st, 2, 0.5, F, chunk, ctypes.byref(steps), F,
                                                  big, N)),
            ("literal_round_refined", lambda: L.literal_round_refined(m, st, 2, 0.5, chunk, N, N, N,
                                                              ctypes.byref(steps), F, big, N)),
            ("literal_round_sampled", lambda: L.literal_round_sampled(m, st, 2, 1.0, F, chunk, N, N, F, big,
                                                              N)),
            ("literal_round_filtered", lambda: L.literal_round_filtered(m, st, 2, N, N, N, N, F, chunk, N, N,
                                                                F, big, N)),
            ("dvs_prefill", lambda: L.dvs_prefill(m, st, 9, 2, F, N, chunk, N, F, big, N))):
        assert call() == -1, name
        assert f"{name}: chunk_keys {chunk}".encode() in L.dvs_last_error()
