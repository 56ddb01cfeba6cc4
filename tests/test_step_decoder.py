"""How a Decoder keeps the workspace of the verification.  On the host, with a library that only looks at its arguments."""
import ctypes

import pytest
import torch

import paper_2507_01663_amd as ra
from paper_2507_01663_amd import binding


class Library:
    """Wants so many bytes; notes the address and the size that each call is given."""

    def __init__(self):
        self.calls = []

    def rollout_attn_verify(self, ctx, verify, at, size, stream):
        at = at.value if isinstance(at, ctypes.c_void_p) else at
        if size < verify.want:
            return ra.RA_ERR_WORKSPACE_TOO_SMALL
        self.calls.append((at, size))
        return ra.RA_OK


class Verify:
    def __init__(self, want):
        self.want = want


@pytest.fixture
def made(monkeypatch):
    """(decoder, library, {address: size} of what it has asked for, a list of what to do while the next block is made)."""
    lib, size, after, empty = Library(), {}, [], torch.empty

    def record(n, dtype=None, device=None):
        t = empty(n, dtype=torch.uint8)
        size[t.data_ptr()] = n
        if after:
            after.pop()()
        return t

    monkeypatch.setattr(torch, "empty", record)
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "rollout_attn_verify_workspace_size", lambda ctx, verify: verify.want)
    monkeypatch.setattr(binding, "rollout_attn_verify", lambda ctx, v, at, n, stream=None: lib.rollout_attn_verify(ctx, v, at, n, stream))
    d = object.__new__(binding.Decoder)
    d.device_ordinal, d.ctx, d._retired, d._raw_stream = 0, 1, [], lambda device: 0
    d.close = lambda: None
    return d, lib, size, after


def kept(d):
    return [t for x in vars(d).values() for t in (x if isinstance(x, list) else [x]) if isinstance(t, torch.Tensor)]


def test_batches_that_creep_leave_few_blocks_behind(made):
    """Every outgrown block is kept, for what is enqueued or captured with it: so a block is at least twice as large as the one that it
    replaces, the blocks of n sizes are no more than log2 of largest over smallest and one, and all together four times what is needed."""
    d, lib, size, _ = made
    wants = list(range(1000, 9000, 7))
    for want in wants:
        d.verify(Verify(want))
    assert len(lib.calls) == len(wants) and all(size[at] >= n >= want for (at, n), want in zip(lib.calls, wants))
    blocks = [t.numel() for t in kept(d)]
    assert len(blocks) <= 5 and sum(blocks) <= 4 * wants[-1], blocks
    assert {at for at, _ in lib.calls} <= {t.data_ptr() for t in kept(d)}


def test_the_first_block_and_much_larger_ones_are_as_large_as_needed(made):
    d, lib, size, _ = made
    for want in (1000, 500, 4000, 1000, 100000):
        d.verify(Verify(want))
    assert [n for _, n in lib.calls] == [1000, 1000, 4000, 4000, 100000] and all(size[at] == n for at, n in lib.calls)


def test_another_thread_s_call_in_between(made):
    """While one call makes its block, a second one makes a smaller one, or a larger one."""
    d, lib, size, after = made
    for first, second in ((9000, 300), (20000, 90000), (200000, 199999)):
        after.append(lambda: d.verify(Verify(second)))
        d.verify(Verify(first))
        for want in (first, second, max(first, second)):
            d.verify(Verify(want))
    assert all(size[at] == n for at, n in lib.calls) and size[d._verify_ws_at[0]] == d._verify_ws_at[1] >= 200000
    assert {at for at, _ in lib.calls} <= {t.data_ptr() for t in kept(d)}
