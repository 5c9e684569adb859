"""GPU: literal_round_filtered called with outputs that do not fit."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_gpu_diffusion import _model_and_state
from tests.test_gpu_model_step import _dev_pools

pytestmark = pytest.mark.gpu


def _make(B):
    w, host, kps, vps = _model_and_state("bf16", B, seed=28)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    return lambda: (dvs.DeviceModel(w, _dev_pools(kps, "bf16"), _dev_pools(vps, "bf16"), "bf16"),
                    dvs.DeviceState(host), host)


def test_refusals():
    B = 2
    m, st, host = _make(B)()
    S, V = host.kv_len.shape[0], m.V
    u = torch.zeros((S, 2 * B + 2), device="cuda")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")   # noqa: E731
    before = st.flat.clone()
    for kw in (dict(accept_out=i32(S - 1)), dict(accept_out=i32(S + 1)),
               dict(logits_out=torch.zeros(S * (B + 1) * V - 1, device="cuda")),
               dict(logits_out=torch.zeros((S, B, V), device="cuda")),
               dict(temperature=torch.ones(S - 1, device="cuda"))):
        with pytest.raises(dvs.DvsError):
            dvs.literal_round_filtered(m, st, B, u, **kw)
    torch.cuda.synchronize()
    assert torch.equal(st.flat, before)
    logits, acc = torch.zeros((S, B + 1, V), device="cuda"), i32(S)
    dvs.literal_round_filtered(m, st, B, u, logits_out=logits, accept_out=acc)
    torch.cuda.synchronize()
    assert int(st.err.item()) == 0 and logits.abs().amax(-1).min() > 0
