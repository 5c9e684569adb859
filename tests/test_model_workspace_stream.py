"""The model's workspace of a call on a given stream is made in that stream's order,
and a replaced one is left to the allocator only after every stream that used it
(no GPU needed: streams, the library and the device checks are stood in for)."""
import contextlib
import types

import torch

from paper_2609_26638_amd import dvs

S, B, V = 3, 4, 11


class Lib:
    need = 1000

    def dvs_filtered_round_workspace_bytes(self, *a):
        return self.need

    def literal_round_filtered(self, *a):
        return 0


def test_workspace_belongs_to_the_calls_stream(monkeypatch):
    streams = [types.SimpleNamespace(cuda_stream=i) for i in range(4)]
    now, made, kept = [streams[0]], [], []

    @contextlib.contextmanager
    def on(s):
        now.append(s)
        yield
        now.pop()

    class Workspace:
        def __init__(self, nbytes, device=None):
            self.nbytes, self.streams = nbytes, set()
            self.buf = types.SimpleNamespace(data_ptr=lambda: 0, record_stream=lambda s: kept.append(
                (nbytes, s.cuda_stream)))
            made.append((nbytes, now[-1].cuda_stream))

    for name, f in (("_dev", lambda t, *a: t), ("_here", lambda *t: None), ("lib", Lib),
                    ("_state_desc", lambda st, e: dvs.DvsState()), ("Workspace", Workspace),
                    ("_stream", lambda s=None: None)):
        monkeypatch.setattr(dvs, name, f)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: now[-1])
    st = types.SimpleNamespace(kv_len=torch.zeros(S), max_pages=4)
    model = types.SimpleNamespace(V=V, ws=None, desc=dvs.DvsModel())

    def call(stream):
        dvs.literal_round_filtered(model, st, B, torch.zeros(S, 2 * B + 2), stream=stream)

    call(streams[1])
    call(streams[1])
    assert made == [(1000, 1)] and kept == []
    call(streams[2])
    call(None)
    call(streams[2])
    assert made == [(1000, 1)] and kept == [(1000, 2), (1000, 0)]
    monkeypatch.setattr(Lib, "need", 2000)
    call(streams[3])
    call(streams[3])
    assert made == [(1000, 1), (2000, 3)] and len(kept) == 2
