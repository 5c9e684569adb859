"""Host-side refusals of the sampling and cache-page calls (no GPU needed:
nothing is launched)."""
import ctypes
import os

import pytest
import torch

from paper_2609_26638_amd import dvs

pytestmark = pytest.mark.skipif(not os.path.exists(dvs.LIB_PATH),
                                reason="libdvs.so not built (run __graft_entry__.build())")
F = ctypes.c_void_p(0x1000)     # never dereferenced: validation fails first
N = None


def _sample(L, logits=F, dtype=0, rows=4, V=8, ld=8, group=1, u=F, token=F):
    return L.sample_filtered(logits, dtype, rows, V, ld, N, N, N, N, group, u, token, N, N, N)


@pytest.mark.parametrize("kw,rc", [
    (dict(logits=N), -1), (dict(u=N), -1), (dict(token=N), -1), (dict(dtype=2), -2),
    (dict(rows=0), -1), (dict(V=0), -1), (dict(V=(1 << 30) + 1, ld=1 << 31), -1), (dict(ld=7), -1),
    (dict(group=0), -1), (dict(group=3), -1)])
def test_sample_filtered_refuses(kw, rc):
    L = dvs.lib()
    assert _sample(L, **kw) == rc
    assert b"sample_filtered" in L.dvs_last_error()


def _accept(L, zv=F, zd=F, vld=8, dld=8, dtype=1, S=2, B=3, V=8, draft=F, width=3, u=F, acc=F,
            tok=F, ws=F, nbytes=1 << 20):
    return L.accept_sampled(zv, 32, vld, zd, 24, dld, dtype, S, B, V, N, N, N, N, draft, width, u,
                            acc, tok, N, ws, nbytes, N)


@pytest.mark.parametrize("kw,rc", [
    (dict(zv=N), -1), (dict(zd=N), -1), (dict(draft=N), -1), (dict(u=N), -1), (dict(acc=N), -1),
    (dict(tok=N), -1), (dict(dtype=5), -2), (dict(S=0), -1), (dict(B=0), -1), (dict(V=0), -1),
    (dict(vld=7), -1), (dict(dld=7), -1), (dict(width=2), -1), (dict(S=1 << 20, B=1 << 12, width=1 << 12), -1),
    (dict(ws=N), -4), (dict(nbytes=16), -4)])
def test_accept_sampled_refuses(kw, rc):
    L = dvs.lib()
    assert _accept(L, **kw) == rc
    assert b"accept_sampled" in L.dvs_last_error()


def test_workspace_queries():
    assert dvs.accept_workspace_bytes(8, 16, 65536) > 0
    assert dvs.accept_workspace_bytes(0, 16, 65536) == 0
    assert dvs.kv_workspace_bytes(64, 5000) > 3 * 4 * 5000
    assert dvs.kv_workspace_bytes(1025, 5000) == 0 and dvs.kv_workspace_bytes(4, 0) == 0


def _state(**kw):
    v = dict(S=4, max_pages=8, num_pool_pages=64, draft_width=3, max_new=16, eos_id=-1)
    v.update({n: 0x1000 for n, _ in dvs.DvsState._fields_[6:]})
    v.update(kw)
    return dvs.DvsState(**v)


def _layers(k=0x1000, v=0x1000, n=2):
    a = (dvs.DvsLayer * n)()
    for l in a:
        l.k_pool, l.v_pool = 0x1000, 0x1000
    a[n - 1].k_pool, a[n - 1].v_pool = k, v
    return a


def _fork(L, st=None, refs=F, layers=None, n_layers=2, heads=2, D=64, dtype=1, n=1, src=F, dst=F,
          window=4, share=1, ws=F, nbytes=1 << 20):
    st = _state() if st is None else st
    layers = _layers() if layers is None else layers
    return L.kv_fork(ctypes.byref(st), refs, layers, n_layers, heads, D, dtype, n, src, dst, window,
                     share, ws, nbytes, N)


@pytest.mark.parametrize("kw,rc", [
    (dict(src=N), -1), (dict(dst=N), -1), (dict(n=0), -1), (dict(n=4), -1), (dict(window=0), -1),
    (dict(refs=N), -1), (dict(dtype=3), -2), (dict(n_layers=0), -1), (dict(heads=0), -1),
    (dict(D=0), -1), (dict(ws=N), -4), (dict(nbytes=64), -4)])
def test_kv_fork_refuses(kw, rc):
    L = dvs.lib()
    assert _fork(L, **kw) == rc
    assert b"kv_fork" in L.dvs_last_error()


@pytest.mark.parametrize("field,value", [
    ("S", 0), ("S", 1025), ("max_pages", 0), ("max_pages", (1 << 20) + 1), ("num_pool_pages", 0),
    ("max_new", 0), ("kv_len", None), ("page_table", None), ("num_pages", None),
    ("free_stack", None), ("free_top", None), ("boundary", None), ("draft", None),
    ("out_tokens", None), ("out_count", None), ("finished", None)])
def test_page_calls_refuse_bad_states(field, value):
    L = dvs.lib()
    st = _state(**{field: value})
    assert _fork(L, st=st) == -1
    assert L.kv_release(ctypes.byref(st), F, 1, F, 4, F, 1 << 20, N) == -1
    assert L.kv_compact(ctypes.byref(st), F, _layers(), 2, 2, 64, 1, N, F, 1 << 20, N) == -1


def test_page_calls_refuse_pools_and_slots():
    L = dvs.lib()
    assert _fork(L, layers=_layers(k=None)) == -1
    assert _fork(L, layers=_layers(v=0x1008)) == -1        # not on 16 bytes
    st = _state()
    assert L.kv_release(ctypes.byref(st), F, 0, F, 4, F, 1 << 20, N) == -1
    assert L.kv_release(ctypes.byref(st), F, 5, F, 4, F, 1 << 20, N) == -1
    assert L.kv_release(ctypes.byref(st), F, 1, N, 4, F, 1 << 20, N) == -1
    assert L.kv_release(ctypes.byref(st), F, 1, F, 0, F, 1 << 20, N) == -1
    assert L.kv_release(ctypes.byref(st), F, 1, F, 4, F, 16, N) == -4
    assert L.kv_compact(ctypes.byref(st), F, None, 2, 2, 64, 1, N, F, 1 << 20, N) == -1


def test_round_refuses():
    L = dvs.lib()
    assert L.literal_round_filtered(None, None, 4, N, N, N, N, F, 256, N, N, F, 1 << 20, N) == -1
    assert b"literal_round_filtered" in L.dvs_last_error()


@pytest.mark.parametrize("vocab,B,rc", [((1 << 22) + 1, 2, -1), (1 << 22, 0, -1), (1 << 22, 4, -1),
                                        (1 << 22, 2, -4)])
def test_round_refuses_models_and_blocks(vocab, B, rc):
    L = dvs.lib()
    layers = (dvs.DvsLayer * 1)()
    for n, _ in dvs.DvsLayer._fields_:
        setattr(layers[0], n, 0x1000)
    m = dvs.DvsModel(0, 1, vocab, 64, 1, 1, 64, 64, 1e4, 1e-6, 0x1000, 0x1000, 0x1000, layers)
    assert (L.dvs_filtered_round_workspace_bytes(ctypes.byref(m), 4, 2, 8, 0) == 0) == (vocab > 1 << 22)
    assert L.literal_round_filtered(ctypes.byref(m), ctypes.byref(_state()), B, N, N, N, N, F, 0, N,
                                    N, F, 16, N) == rc
    assert b"literal_round_filtered" in L.dvs_last_error()


def test_binding_refuses_host_tensors():
    z, u = torch.zeros(2, 8), torch.zeros(2)
    with pytest.raises(dvs.DvsError, match="logits"):
        dvs.sample_filtered(z, u)
    with pytest.raises(dvs.DvsError, match="z_verify"):
        dvs.accept_sampled(torch.zeros(1, 2, 8), torch.zeros(1, 1, 8), torch.zeros(1, 1), u)
    with pytest.raises(dvs.DvsError):
        dvs.KVPools([], [])
    with pytest.raises(dvs.DvsError):
        dvs.KVPools([torch.zeros(4, 2, 16, 64)], [torch.zeros(4, 2, 64, 16)])
