"""Pools, workspaces and outputs of the sampling and cache-page calls: on another
device than the current one, or empty, they are refused before the library is
called (no GPU needed: tensors and the device are stood in for)."""
import types

import pytest
import torch

from paper_2609_26638_amd import dvs


class Tensor:
    """On device `dev`, with `n` entries."""

    def __init__(self, dev, n=4):
        self.dev, self.shape, self.device = dev, (n,), f"cuda:{dev}"

    def get_device(self):
        return self.dev

    def numel(self):
        return self.shape[0]

    def data_ptr(self):
        return 0x1000


@pytest.fixture(autouse=True)
def _one_device(monkeypatch):
    lib = types.SimpleNamespace(dvs_kv_workspace_bytes=lambda *a: 256,
                                dvs_accept_workspace_bytes=lambda *a: 256)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(dvs, "_dev", lambda t, *a: t)
    monkeypatch.setattr(dvs, "lib", lambda: lib)      # has none of the calls themselves


def _state(dev=0):
    return types.SimpleNamespace(kv_len=Tensor(dev), pool_pages=8)


def _pools(dev=0):
    return types.SimpleNamespace(pages=8, keep=([Tensor(dev)], [Tensor(dev)]))


def _ws(dev):
    return types.SimpleNamespace(buf=Tensor(dev))


IDS = Tensor(0)


@pytest.mark.parametrize("call", [
    lambda: dvs.kv_fork(_state(), _pools(1), IDS, IDS, 4),
    lambda: dvs.kv_fork(_state(), _pools(), IDS, IDS, 4, workspace=_ws(1)),
    lambda: dvs.kv_release(_state(), IDS, 4, workspace=_ws(1)),
    lambda: dvs.kv_compact(_state(), _pools(1), moved_out=Tensor(0, 1)),
    lambda: dvs.kv_compact(_state(), _pools(), moved_out=Tensor(1, 1)),
    lambda: dvs.kv_compact(_state(), _pools(), moved_out=Tensor(0, 1), workspace=_ws(1))])
def test_another_device(call):
    with pytest.raises(dvs.DvsError, match="current device"):
        call()


def test_empty_moved_out():
    with pytest.raises(dvs.DvsError, match="moved_out"):
        dvs.kv_compact(_state(), _pools(), moved_out=Tensor(0, 0))


def test_pools_on_two_devices():
    k, v = torch.zeros(4, 2, 16, 8), torch.zeros(4, 2, 8, 16)
    dvs.KVPools([k, k], [v, v])
    for kk, vv in (([k, k.to("meta")], [v, v]), ([k, k], [v, v.to("meta")])):
        with pytest.raises(dvs.DvsError, match="one device"):
            dvs.KVPools(kk, vv)


def test_empty_error_word():
    with pytest.raises(dvs.DvsError, match="err"):
        dvs._check_err(Tensor(0, 0))
    dvs._check_err(None)
    dvs._check_err(Tensor(0, 1))
