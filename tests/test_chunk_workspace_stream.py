"""Workspaces come from the memory of the stream that the call is given: a block that another stream gave back may still be read by
what is enqueued there.  On the host, with a library that only looks at its arguments."""
import contextlib

import pytest
import torch

import paper_2507_01663_amd as ra
from paper_2507_01663_amd import binding


class Stream:
    cuda_stream = 77


class Library:
    def rollout_attn_extend(self, *args):
        return ra.RA_OK

    rollout_attn_decode = rollout_attn_extend


@pytest.mark.parametrize("call", ["extend", "decode"])
@pytest.mark.parametrize("stream", [None, Stream()])
def test_a_workspace_is_its_stream_s(monkeypatch, call, stream):
    at, made, empty = [None], [], torch.empty

    @contextlib.contextmanager
    def on(s):
        was, at[0] = at[0], s
        yield
        at[0] = was

    def record(n, dtype=None, device=None):
        made.append(at[0])
        return empty(n, dtype=torch.uint8)

    monkeypatch.setattr(torch, "empty", record)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(binding, "load_library", lambda: Library())
    for name in ("rollout_attn_extend", "rollout_attn_decode"):
        monkeypatch.setattr(binding, name, lambda *args: None)
        monkeypatch.setattr(binding, name + "_workspace_size" if name.endswith("extend") else "rollout_attn_workspace_size", lambda ctx, desc: 5000)
    d = object.__new__(binding.Decoder)
    d.device_ordinal, d.ctx, d._retired, d._raw_stream, d._ws, d._ws_at, d._chunk_ws_at = 0, 1, [], lambda device: 0, None, None, None
    d.close = lambda: None
    getattr(d, call)(None, stream=stream)
    getattr(d, call)(None, stream=stream)
    assert made == [stream] and at == [None]
