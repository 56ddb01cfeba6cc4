"""How a Decoder keeps the workspace of the attention of chunks: the library is told the size of the memory that it is given, also
where another thread's call replaces the tensor in between.  On the host, with a library that only looks at its arguments."""
import ctypes

import torch

import paper_2507_01663_amd as ra
from paper_2507_01663_amd import binding


class Tensors:
    """Stands in for torch.empty; remembers what lies where."""

    def __init__(self, monkeypatch):
        self.size, self.after, self.made = {}, None, torch.empty
        monkeypatch.setattr(torch, "empty", self.empty)

    def empty(self, n, dtype=None, device=None):
        t = self.made(n, dtype=torch.uint8)
        self.size[t.data_ptr()] = n
        after, self.after = self.after, None
        if after:
            after()
        return t


class Library:
    """Wants so many bytes; every call notes the address and the size that it is given."""

    def __init__(self):
        self.calls = []

    def rollout_attn_extend(self, ctx, extend, at, size, stream):
        at = at.value if isinstance(at, ctypes.c_void_p) else at
        if size < extend.want:
            return ra.RA_ERR_WORKSPACE_TOO_SMALL
        self.calls.append((at, size))
        return ra.RA_OK


class Extend:
    def __init__(self, want):
        self.want = want


def decoder(monkeypatch):
    lib = Library()
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "rollout_attn_extend_workspace_size", lambda ctx, extend: extend.want)
    monkeypatch.setattr(binding, "rollout_attn_extend", lambda ctx, e, at, size, stream=None: lib.rollout_attn_extend(ctx, e, at, size, stream))
    d = object.__new__(binding.Decoder)
    d.device_ordinal, d.ctx, d._retired, d._raw_stream = 0, 1, [], lambda device: 0
    d._ws = d._ws_at = d._chunk_ws_at = None
    d.close = lambda: None
    return d, lib


def test_the_workspace_grows_and_is_kept(monkeypatch):
    tensors = Tensors(monkeypatch)
    d, lib = decoder(monkeypatch)
    for want in (1000, 500, 0, 4000, 1000):
        d.extend(Extend(want))
    sizes = [size for _, size in lib.calls]
    assert sizes == [1000, 1000, 1000, 4000, 4000] and all(tensors.size[at] >= size for at, size in lib.calls)


def test_another_thread_s_call_in_between(monkeypatch):
    """While one call makes its tensor, a second one makes a smaller one, or a larger one."""
    for first, second in ((9000, 300), (300, 9000), (9000, 8999)):
        tensors = Tensors(monkeypatch)
        d, lib = decoder(monkeypatch)
        tensors.after = lambda: d.extend(Extend(second))
        d.extend(Extend(first))
        for want in (first, second, max(first, second)):
            d.extend(Extend(want))
        assert len(lib.calls) == 5 and all(tensors.size[at] >= size for at, size in lib.calls)
        assert d._chunk_ws_at[1] == max(first, second) == tensors.size[d._chunk_ws_at[0]]
        held = {t.data_ptr() for x in vars(d).values() for t in (x if isinstance(x, list) else [x]) if isinstance(t, torch.Tensor)}
        assert {at for at, _ in lib.calls} <= held           # (nothing that was enqueued loses its memory)
