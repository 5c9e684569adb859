"""literal_round_filtered refuses outputs that do not fit before it takes a
workspace or calls the library (no GPU needed: the device checks are stood in
for)."""
import types

import pytest
import torch

from paper_2609_26638_amd import dvs

S, B, V = 3, 4, 11


def _call(monkeypatch, **kw):
    called = []
    monkeypatch.setattr(dvs, "_dev", lambda t, *a: t)
    monkeypatch.setattr(dvs, "_here", lambda *t: None)
    monkeypatch.setattr(dvs, "lib", lambda: called.append(1) or pytest.fail("reached the library"))
    st = types.SimpleNamespace(kv_len=torch.zeros(S), max_pages=4)
    model = types.SimpleNamespace(V=V, ws=None, desc=None)
    with pytest.raises(dvs.DvsError) as e:
        dvs.literal_round_filtered(model, st, B, torch.zeros(S, 2 * B + 2), **kw)
    assert model.ws is None and not called
    return str(e.value)


@pytest.mark.parametrize("n", [0, S * (B + 1) * V - 1, S * B * V, S * (B + 1) * V + 1])
def test_logits_out(monkeypatch, n):
    assert "logits_out" in _call(monkeypatch, logits_out=torch.zeros(n))


@pytest.mark.parametrize("n", [0, S - 1, S + 1])
def test_accept_out(monkeypatch, n):
    assert "accept_out" in _call(monkeypatch, accept_out=torch.zeros(n, dtype=torch.int32))
