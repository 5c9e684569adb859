"""GPU: calls on a stream that is not the current one, which has work of its own:
workspaces and outputs that a call makes belong to the call's stream."""
import numpy as np
import pytest
import torch

from paper_2609_26638_amd import dvs, synth

pytestmark = pytest.mark.gpu


def _busy():
    """Some milliseconds of work for the current stream, over memory that it frees."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(20):
        a = a @ a * 1e-4
    junk = [torch.full((1 << 18,), 7, dtype=torch.int32, device="cuda") for _ in range(8)]
    return a, junk[0]


def _bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).view(torch.bfloat16).cuda()


@pytest.mark.parametrize("chunk", [0, 64])
def test_attention(chunk):
    B = 8
    ai = synth.make_attn_inputs(0, 3, [900, 45, 310], B, B, 16, 4, 128, "bf16", scatter=True)
    t = [_bf16(getattr(ai, n)) for n in ("q", "k_new", "v_new", "k_pool", "v_pool")]
    st = dvs.DeviceState(ai.state)
    call = lambda **kw: dvs.attn_hybrid_block(*t, st.page_table, st.kv_len, B, B, ai.scale,   # noqa: E731
                                              err=st.err, chunk_keys=chunk, **kw)
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = dvs.Workspace(256)
    for kw in ({}, dict(workspace=ws), dict(workspace=ws)):
        keep = _busy()
        got = call(stream=s, **kw)
        keep = _busy()
        s.synchronize()
        assert torch.equal(got, want) and int(st.err.item()) == 0
        torch.cuda.synchronize()
    del keep


def test_top1():
    B = 6
    li = synth.make_logit_inputs(0, 4, B, B, 40000, 4.0, 0.9)
    logits, draft = _bf16(li.logits), torch.from_numpy(li.draft).cuda()
    want = dvs.argmax_accept(logits, B, draft) + dvs.top1_confidence(logits)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(2):
        keep = _busy()
        got = dvs.argmax_accept(logits, B, draft, stream=s)
        got += dvs.top1_confidence(logits, stream=s)
        keep = _busy()
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        torch.cuda.synchronize()
    del keep
