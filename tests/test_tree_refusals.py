"""Host-side refusals of the tree step's calls (no GPU needed: nothing is
launched)."""
import ctypes
import os
import types

import pytest
import torch

from paper_2609_26638_amd import dvs

needs_lib = pytest.mark.skipif(not os.path.exists(dvs.LIB_PATH),
                               reason="libdvs.so not built (run __graft_entry__.build())")
F = ctypes.c_void_p(0x1000)     # never dereferenced: validation fails first
N = None


@needs_lib
@pytest.mark.parametrize("kw", [dict(parent=N), dict(mask=N), dict(S=0), dict(R=0), dict(R=1025),
                                dict(mask=ctypes.c_void_p(0x1004), R=33)])
def test_tree_masks_refuses(kw):
    a = dict(parent=F, S=2, R=4, mask=F, depth=N, err=N, stream=N) | kw
    assert dvs.lib().tree_masks(*a.values()) == -1
    assert b"tree_masks" in dvs.lib().dvs_last_error()


def _append(**kw):
    a = dict(q=F, q_seq=512, q_ld=256, k=F, k_seq=256, k_ld=128, v=F, v_seq=256, v_ld=128, kp=F,
             vp=F, table=F, kv_len=F, depth=N, S=2, R=2, Hq=4, Hkv=2, D=64, rot=64, theta=1e4,
             max_pages=4, pool=8, dtype=1, q_out=ctypes.c_void_p(0x9000), err=N, stream=N) | kw
    return dvs.lib().kv_append_rope(*a.values())


@needs_lib
@pytest.mark.parametrize("kw,rc", [
    (dict(k=N), -1), (dict(v=N), -1), (dict(kp=N), -1), (dict(vp=N), -1), (dict(table=N), -1),
    (dict(kv_len=N), -1), (dict(q=N), -1), (dict(q_out=N), -1), (dict(S=0), -1), (dict(R=0), -1),
    (dict(Hkv=0), -1), (dict(Hq=0), -1), (dict(D=80), -2), (dict(rot=24), -2), (dict(rot=-16), -2),
    (dict(rot=80), -2), (dict(theta=0.0), -1), (dict(theta=float("inf")), -1),
    (dict(theta=float("nan")), -1), (dict(dtype=2), -2), (dict(max_pages=0), -1), (dict(pool=0), -1),
    (dict(q_ld=255), -1), (dict(k_ld=127), -1), (dict(v_ld=0), -1),
    (dict(q_out=F, q_ld=300, q_seq=600), -1), (dict(kp=ctypes.c_void_p(0x1008)), -1),
    (dict(q=ctypes.c_void_p(0x1001)), -1), (dict(v=ctypes.c_void_p(0x1002), dtype=0), -1),
    (dict(S=1 << 20, R=1 << 16), -2)])
def test_kv_append_rope_refuses(kw, rc):
    assert _append(**kw) == rc
    assert b"kv_append_rope" in dvs.lib().dvs_last_error()


def _attn(**kw):
    a = dict(q=F, kp=F, vp=F, table=F, kv_len=F, mask=F, S=2, R=4, Hq=4, Hkv=2, D=64, max_pages=4,
             pool=8, scale=0.1, dtype=1, out=F, err=N, ws=F, nbytes=1 << 30, stream=N) | kw
    return dvs.lib().attn_tree(*a.values())


@needs_lib
@pytest.mark.parametrize("kw,rc", [
    (dict(q=N), -1), (dict(kp=N), -1), (dict(vp=N), -1), (dict(table=N), -1), (dict(kv_len=N), -1),
    (dict(out=N), -1), (dict(S=0), -1), (dict(R=0), -1), (dict(R=1025), -1), (dict(Hq=5), -1),
    (dict(Hkv=0), -1), (dict(D=32), -2), (dict(max_pages=0), -1), (dict(pool=0), -1),
    (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(dtype=3), -2), (dict(ws=N), -4),
    (dict(nbytes=16), -4), (dict(q=ctypes.c_void_p(0x1008)), -1),
    (dict(vp=ctypes.c_void_p(0x1004)), -1), (dict(out=ctypes.c_void_p(0x1002)), -1),
    (dict(ws=ctypes.c_void_p(0x1080)), -1), (dict(Hq=1 << 20, Hkv=1, R=2), -2),
    (dict(max_pages=1 << 28), -2)])
def test_attn_tree_refuses(kw, rc):
    assert _attn(**kw) == rc
    assert b"attn_tree" in dvs.lib().dvs_last_error()


def _state(**kw):
    v = dict(S=4, max_pages=8, num_pool_pages=64, draft_width=3, max_new=16, eos_id=-1)
    v.update({n: 0x1000 for n, _ in dvs.DvsState._fields_[6:]})
    v.update(kw)
    return dvs.DvsState(**v)


def _commit(layer=None, **kw):
    layers = (dvs.DvsLayer * 2)()
    for x in layers:
        x.k_pool = x.v_pool = 0x1000
    for f, v in (layer or {}).items():
        setattr(layers[1], f, v)
    a = dict(st=ctypes.byref(_state()), layers=layers, n=2, heads=2, D=64, dtype=1, R=4, parent=F,
             tokens=F, argmax=F, acc=N, path=N, ws=F, nbytes=1 << 20, stream=N) | kw
    return dvs.lib().accept_commit_tree(*a.values())


@needs_lib
@pytest.mark.parametrize("kw,rc", [
    (dict(st=N), -1), (dict(layers=N), -1), (dict(n=0), -1), (dict(heads=0), -1), (dict(D=48), -2),
    (dict(dtype=9), -2), (dict(R=0), -1), (dict(R=1025), -1), (dict(parent=N), -1),
    (dict(tokens=N), -1), (dict(argmax=N), -1), (dict(ws=N), -4), (dict(nbytes=64), -4),
    (dict(layer=dict(v_pool=None)), -1), (dict(layer=dict(k_pool=0x1008)), -1)])
def test_accept_commit_tree_refuses(kw, rc):
    assert _commit(**kw) == rc
    assert b"accept_commit_tree" in dvs.lib().dvs_last_error()


@needs_lib
@pytest.mark.parametrize("kw", [dict(S=0), dict(S=1025), dict(kv_len=None), dict(page_table=None),
                                dict(finished=None), dict(max_pages=0), dict(num_pool_pages=0),
                                dict(num_pages=None), dict(free_top=None), dict(max_new=0)])
def test_accept_commit_tree_refuses_states(kw):
    st = _state(**kw)
    assert _commit(st=ctypes.byref(st)) == -1
    assert b"accept_commit_tree" in dvs.lib().dvs_last_error()


@needs_lib
def test_workspace_queries():
    f, b = dvs.tree_workspace_bytes, torch.bfloat16
    assert f(8, 32, 16, 4, 128, 130, b) > 0 and f(8, 32, 16, 4, 128, 130, torch.float32) > 0
    for bad in ((0, 32, 16, 4, 128, 130), (8, 0, 16, 4, 128, 130), (8, 1025, 16, 4, 128, 130),
                (8, 32, 15, 4, 128, 130), (8, 32, 16, 0, 128, 130), (8, 32, 16, 4, 100, 130),
                (8, 32, 16, 4, 128, 0)):
        assert f(*bad, b) == 0
    assert f(8, 32, 16, 4, 128, 130, 7) == 0
    assert dvs.accept_tree_workspace_bytes(8, 64) >= 8 * 64 * 8
    for bad in ((0, 4), (1025, 4), (4, 0), (4, 1025)):
        assert dvs.accept_tree_workspace_bytes(*bad) == 0


# ---- the binding's own checks: tensors and the device are stood in for

class Tensor:
    def __init__(self, *shape, dev=0, stride=None):
        self.shape, self.dev, self.device, self.is_cuda = shape, dev, f"cuda:{dev}", True
        self.dtype = torch.bfloat16
        self._stride = stride

    def dim(self):
        return len(self.shape)

    def stride(self):
        if self._stride:
            return self._stride
        n, out = 1, []
        for x in reversed(self.shape):
            out.append(n)
            n *= x
        return tuple(reversed(out))

    def get_device(self):
        return self.dev

    def numel(self):
        return 1 << 20

    def data_ptr(self):
        return 0x1000


@pytest.fixture
def _one_device(monkeypatch):
    lib = types.SimpleNamespace(dvs_tree_workspace_bytes=lambda *a: 256,
                                dvs_accept_tree_workspace_bytes=lambda *a: 256)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(dvs, "_dev", lambda t, *a: t)
    monkeypatch.setattr(torch, "Tensor", Tensor)      # _rows looks at the class
    monkeypatch.setattr(dvs, "lib", lambda: lib)      # has none of the calls themselves


S, R, Hq, Hkv, D, P = 2, 3, 4, 2, 64, 9


def _append_args(**kw):
    a = dict(q=Tensor(S, R, Hq, D), k_new=Tensor(S, R, Hkv, D), v_new=Tensor(S, R, Hkv, D),
             k_pool=Tensor(P, Hkv, 16, D), v_pool=Tensor(P, Hkv, D, 16), page_table=Tensor(S, 5),
             kv_len=Tensor(S), depth=Tensor(S, R), q_out=Tensor(S, R, Hq, D))
    return a | kw


@pytest.mark.parametrize("kw,match", [
    (dict(v_pool=Tensor(P, Hkv, 16, D)), "pools"), (dict(v_new=Tensor(S, R, Hq, D)), "k_new"),
    (dict(q=Tensor(S, R + 1, Hq, D)), "q must be"), (dict(q=Tensor(S, R, Hq, 96)), "q must be"),
    (dict(q=Tensor(S, R, Hq, D, stride=(768, 256, 1, 4))), "side by side"),
    (dict(q=Tensor(S, R, Hq, D, stride=(768, 256, 128, 1))), "side by side"),
    (dict(q_out=Tensor(S, R, Hkv, D)), "q_out"), (dict(q=None), "q_out without q"),
    (dict(depth=Tensor(S, R + 1)), "depth"), (dict(page_table=Tensor(S + 1, 5)), "S rows"),
    (dict(kv_len=Tensor(1)), "S rows"), (dict(k_pool=Tensor(P, Hkv, 16, D, dev=1)), "current device"),
    (dict(depth=Tensor(S, R, dev=1)), "current device"), (dict(err=Tensor(0)), "err"),
    (dict(q_out=Tensor(S, R, Hq, D, dev=1)), "current device")])
def test_append_binding(_one_device, kw, match):
    with pytest.raises(dvs.DvsError, match=match):
        dvs.kv_append_rope(**_append_args(**kw))


@pytest.mark.parametrize("kw,match", [
    (dict(q=Tensor(S, R, Hq, 96)), "head size"), (dict(mask=Tensor(S, R, 2)), "mask"),
    (dict(mask=Tensor(S, R, 1, dev=1)), "current device"), (dict(out=Tensor(S, R, Hkv, D)), "out"),
    (dict(workspace=types.SimpleNamespace(buf=Tensor(9, dev=1))), "current device"),
    (dict(kv_len=Tensor(3)), "S rows")])
def test_attn_binding(_one_device, kw, match):
    a = dict(q=Tensor(S, R, Hq, D), k_pool=Tensor(P, Hkv, 16, D), v_pool=Tensor(P, Hkv, D, 16),
             page_table=Tensor(S, 5), kv_len=Tensor(S), mask=Tensor(S, R, 1), softmax_scale=0.1,
             out=Tensor(S, R, Hq, D), workspace=types.SimpleNamespace(buf=Tensor(9))) | kw
    with pytest.raises(dvs.DvsError, match=match):
        dvs.attn_tree(**a)


@pytest.mark.parametrize("kw,match", [
    (dict(tokens=Tensor(S, R + 1)), "parent, tokens"), (dict(argmax=Tensor(S + 1, R)), "parent"),
    (dict(accept_out=Tensor(S + 1)), "accept_out"), (dict(path_out=Tensor(S, R + 1)), "path_out"),
    (dict(tokens=Tensor(S, R, dev=1)), "current device"),
    (dict(workspace=types.SimpleNamespace(buf=Tensor(9, dev=1))), "current device")])
def test_commit_binding(_one_device, kw, match):
    pools = types.SimpleNamespace(pages=P, keep=([Tensor(P)], [Tensor(P)]))
    a = dict(st=types.SimpleNamespace(kv_len=Tensor(S), pool_pages=P), pools=pools,
             parent=Tensor(S, R), tokens=Tensor(S, R), argmax=Tensor(S, R), accept_out=Tensor(S),
             path_out=Tensor(S, R), workspace=types.SimpleNamespace(buf=Tensor(9))) | kw
    with pytest.raises(dvs.DvsError, match=match):
        dvs.accept_commit_tree(**a)


@pytest.mark.parametrize("kw,match", [
    (dict(mask_out=Tensor(S, R, 2)), "mask_out"), (dict(depth_out=Tensor(S)), "depth_out"),
    (dict(parent=Tensor(S, R, dev=1)), "current device"), (dict(err=Tensor(0)), "err")])
def test_masks_binding(_one_device, kw, match):
    a = dict(parent=Tensor(S, R), mask_out=Tensor(S, R, 1), depth_out=Tensor(S, R)) | kw
    with pytest.raises(dvs.DvsError, match=match):
        dvs.tree_masks(**a)
