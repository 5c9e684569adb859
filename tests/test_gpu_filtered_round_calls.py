"""GPU: literal_round_filtered called on a stream of its own, with a workspace that
grows on another, and with outputs that do not fit."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs
from tests.test_gpu_diffusion import _model_and_state
from tests.test_gpu_model_step import _dev_pools, _states_equal

pytestmark = pytest.mark.gpu


def _make(B):
    w, host, kps, vps = _model_and_state("bf16", B, seed=28)
    host.draft = np.zeros((host.kv_len.shape[0], B), np.int32)
    return lambda: (dvs.DeviceModel(w, _dev_pools(kps, "bf16"), _dev_pools(vps, "bf16"), "bf16"),
                    dvs.DeviceState(host), host)


def _busy():
    """Some milliseconds of work for the current stream."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(20):
        a = a @ a * 1e-4
    return a


def test_explicit_streams():
    """A fresh model on a stream of its own beside work of the current one, then on
    a second stream, then on a third with a workspace that replaces the first."""
    B = 6
    fresh = _make(B)
    m, st, host = fresh()
    S = host.kv_len.shape[0]
    gen = torch.Generator(device="cuda").manual_seed(3)
    u = [torch.rand((S, 2 * B + 2), device="cuda", generator=gen) for _ in range(4)]
    par = dict(top_k=torch.full((S,), 30, dtype=torch.int32, device="cuda"),
               top_p=torch.full((S,), 0.9, device="cuda"))
    chunks = (256, 256, 64, 64)
    for i, c in enumerate(chunks):
        dvs.literal_round_filtered(m, st, B, u[i], chunk_keys=c, **par)
    torch.cuda.synchronize()
    assert int(st.err.item()) == 0
    want = st.to_host(host)
    streams = [torch.cuda.Stream() for _ in chunks]
    m, st, _ = fresh()
    torch.cuda.synchronize()
    seen = set()
    for i, c in enumerate(chunks):
        keep = _busy()
        dvs.literal_round_filtered(m, st, B, u[i], chunk_keys=c, stream=streams[i], **par)
        seen.add((m.ws.nbytes, m.ws.buf.data_ptr()))
        junk = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]
        if i + 1 < len(chunks):
            streams[i + 1].wait_stream(streams[i])
    assert len(seen) == 2                          # grown once
    streams[-1].synchronize()
    assert int(st.err.item()) == 0
    _states_equal(st, want)
    del keep, junk


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
