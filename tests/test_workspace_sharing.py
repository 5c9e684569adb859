"""A workspace that attn_hybrid_block shares with calls that leave anything in it (the device and the
library are stood in for)."""
import types

import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_tree_refusals import D, Hkv, Hq, P, R, S, Tensor


@pytest.fixture
def _stubs(monkeypatch):
    lib = types.SimpleNamespace(attn_tree=lambda *a: 0, accept_commit_tree=lambda *a: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(dvs, "_dev", lambda t, *a: t)
    monkeypatch.setattr(dvs, "_stream", lambda *a: 0)
    monkeypatch.setattr(dvs, "_state_desc", lambda *a: dvs.DvsState())
    monkeypatch.setattr(dvs, "_check_pools", lambda *a: None)
    monkeypatch.setattr(dvs, "lib", lambda: lib)


def attn_tree(ws):
    dvs.attn_tree(Tensor(S, R, Hq, D), Tensor(P, Hkv, 16, D), Tensor(P, Hkv, D, 16), Tensor(S, 5),
                  Tensor(S), None, 0.1, out=Tensor(S, R, Hq, D), workspace=ws)


def accept_commit_tree(ws):
    st = types.SimpleNamespace(kv_len=Tensor(S))
    pools = types.SimpleNamespace(keep=([Tensor(P)], [Tensor(P)]), layers=(dvs.DvsLayer * 1)(),
                                  n_kv_heads=Hkv, head_dim=D, dtype=1)
    t = Tensor(S, R)
    dvs.accept_commit_tree(st, pools, t, t, t, accept_out=Tensor(S), path_out=t, workspace=ws)


def scratch(ws):     # of accept_sampled and the page calls
    assert dvs._scratch(ws, 16, "cuda:0", None) is ws.buf


@pytest.mark.parametrize("call", [attn_tree, accept_commit_tree, scratch])
def test_a_lent_workspace_is_cleared_before_it_counts_again(_stubs, call):
    ws = types.SimpleNamespace(buf=Tensor(9), shape=("attn", 1))
    call(ws)
    assert ws.shape is None
