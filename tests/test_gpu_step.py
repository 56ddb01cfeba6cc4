"""Whole steps: places of the new tokens, their keys and values into the cache, attention, verification of the drafts, the new lengths,
with nothing of it on the host; recorded into a graph, and beside other streams' calls."""
import numpy as np
import pytest
import torch

import paper_2507_01663_amd as ra
import step_util as su
from chunk_util import Cache
from gpu_util import context
from step_util import DEV, PAGE, Placing, Releasing, batch, drafting, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", params=["binary64 sums", "binary32 sums first"])
def dec(request):
    d = context() if request.param == "binary64 sums" else context(VERIFY_FEW=0)
    yield d
    d.close()


def capture(fn):
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        fn()
    return g


class Loop:
    """A batch that writes on, n tokens a sequence looked at in a step: one that is sure and n - 1 guesses.  The buffers that a step reads
    and writes are always the same."""

    def __init__(self, dec, seqs, n, V=700, pages=200, Hq=4, Hkv=2, D=64, seed=0):
        self.dec, self.seqs, self.n, self.V = dec, seqs, n, V
        R = seqs * n
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        zeros = lambda *s, kind=torch.int32: torch.zeros(s, dtype=kind, device=DEV)
        self.lens, self.held, self.after, self.accepted, self.next = (zeros(seqs) for _ in range(5))
        self.table, self.cu, self.new = zeros(seqs, 12) - 1, zeros(seqs + 1), zeros(seqs) + n
        self.stack = torch.randperm(pages, generator=self.g, device=DEV).to(torch.int32)
        self.free = zeros(1) + pages
        self.positions, self.slots, self.tokens, self.out = zeros(R), zeros(R, kind=torch.int64), zeros(R), zeros(R)
        self.q, self.k, self.v = (zeros(R, h, D, kind=torch.bfloat16) for h in (Hq, Hkv, Hkv))
        self.o, self.lse = zeros(R, Hq, D, kind=torch.bfloat16), zeros(R, Hq, kind=torch.float32)
        self.kp, self.vp = (zeros(pages, Hkv, PAGE, D, kind=torch.bfloat16) for _ in range(2))
        self.logits, self.u, self.w = zeros(R, V, kind=torch.float32), zeros(R, kind=torch.float32), zeros(seqs, kind=torch.float32)
        self.place = ra.place_from_tensors(self.lens, self.new, self.held, self.table, self.stack, self.free, self.cu, self.after, self.held, self.free,
                                           self.positions, self.slots)
        self.append = ra.append_chunk_from_tensors(self.k, self.v, self.cu, n, self.table, self.lens, self.kp, self.vp)
        self.extend = ra.extend_from_tensors(self.q, self.kp, self.vp, self.cu, n, self.table, self.after, self.o, self.lse, D ** -0.5)
        self.verify = ra.verify_from_tensors(self.logits, self.cu, self.tokens, self.u, self.w, self.accepted, self.out, None, self.next)

    def state(self):
        return [self.lens, self.held, self.table, self.stack, self.free, self.kp, self.vp, self.accepted, self.next, self.out, self.o, self.slots, self.positions]

    def inputs(self, step):
        """What the layers around would have computed, the random numbers and the guesses: the step's, whoever asks."""
        g = torch.Generator(device=DEV).manual_seed(1000 + step)
        for t in (self.q, self.k, self.v, self.logits):
            t.normal_(generator=g)
        self.logits.mul_(2.0)
        for t in (self.u, self.w):
            t.uniform_(generator=g)
        self.tokens.random_(0, self.V, generator=g)
        # most guesses are the likeliest token
        right = torch.rand(self.tokens.shape, generator=g, device=DEV) < 0.8
        best = torch.cat([self.logits.argmax(1)[-1:], self.logits.argmax(1)[:-1]]).to(torch.int32)
        self.tokens.copy_(torch.where(right, best, self.tokens))
        self.logits.view(-1)[torch.arange(self.logits.shape[0], device=DEV) * self.V + self.logits.argmax(1)] += 6.0

    def step(self):
        self.dec.place(self.place)
        self.dec.append_chunk(self.append)
        self.dec.extend(self.extend)
        self.dec.verify(self.verify)
        self.lens.add_(self.accepted).add_(1)


def test_steps_replayed_from_a_graph(dec):
    """Ten replays, each against the same step of a batch that is run call by call; and the counts against the plain form."""
    a, b = Loop(dec, 9, 4), Loop(dec, 9, 4)
    a.inputs(0), b.inputs(0)
    a.step()                                                 # (the decoder's workspaces exist before the capture)
    a2 = Loop(dec, 9, 4)
    a2.inputs(0)
    torch.cuda.synchronize()
    graph = capture(a2.step)
    seen = set()
    for i in range(10):
        for x in (a2, b):
            x.inputs(i)
        before = b.lens.clone()
        torch.cuda.synchronize()
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in zip(a2.state(), b.state()):
            assert torch.equal(x, y), i
        want = su.verify(b.logits.double().cpu().numpy(), b.cu.tolist(), b.tokens.tolist(), b.u.double().tolist(), b.w.double().tolist())
        assert b.accepted.tolist() == want[0] and b.next.tolist() == want[3] and b.out.tolist() == want[1]
        assert (b.lens == before + b.accepted + 1).all()
        seen |= set(want[0])
    assert len(seen) >= 3                                    # (drafts of all lengths stayed)
    used = [p for row, h in zip(b.table.tolist(), b.held.tolist()) for p in row[:h]]
    assert sorted(used + b.stack[:int(b.free)].tolist()) == list(range(b.stack.numel()))
    # the cache holds what was appended: the keys of a step's tokens are where the slots say
    page, slot = b.slots // PAGE, b.slots % PAGE
    assert torch.equal(b.kp[page, :, slot], b.k)


def test_a_captured_step_has_room_for_more_tokens(dec):
    """Sequences that end ask for none from then on: the offsets shrink, and the places behind them are -1, which the append leaves out."""
    x = Loop(dec, 6, 3)
    x.inputs(0)
    x.step()
    torch.cuda.synchronize()
    graph = capture(x.step)
    for i, alive in enumerate([[1] * 6, [1, 0, 1, 1, 0, 1], [0, 0, 0, 1, 0, 0], [0] * 6]):
        x.inputs(i)
        x.new.copy_(ints(np.array(alive) * 3))
        before = x.lens.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        total = 3 * sum(alive)
        assert x.cu.tolist() == [0] + np.cumsum(np.array(alive) * 3).tolist()
        assert (x.positions[total:] == -1).all() and (x.slots[total:] == -1).all() and (x.positions[:total] >= 0).all()
        for b, on in enumerate(alive):
            # (a sequence without rows has accepted none; the loop's one more is for it to take back)
            assert int(x.accepted[b]) == 0 or on
            if not on:
                assert int(x.next[b]) == -1
                x.lens[b] = before[b]


@pytest.mark.parametrize("what", ["place", "release", "verify", "verify drafts"])
def test_each_call_replayed_from_a_graph(dec, what):
    """Other inputs in the same buffers at every replay, the program's own work between them."""
    def make(seed):
        if what == "place":
            lens, asked, held, table, stack, free, groups = batch(seed, 1300, group=4, prefix=2)
            M = 40
            table = np.concatenate([table, np.full((1300, M - table.shape[1]), -1, dtype=np.int32)], axis=1)
            stack = np.concatenate([stack, np.full(20000 - len(stack), -1)])
            return Placing(lens, asked, held, table, stack, free, 80000, [g if i < 2 else np.concatenate([g, np.zeros(3000 - len(g))]) for i, g in enumerate(groups)])
        if what == "release":
            lens, asked, held, table, stack, free, groups = batch(seed, 1300)
            table = np.concatenate([table, np.full((1300, 40 - table.shape[1]), -1, dtype=np.int32)], axis=1)
            return Releasing(lens // 2, held, table, np.concatenate([stack, np.full(50000 - len(stack), -1)]), free)
        return drafting(seed, [3, 1, 0, 4, 2], 9001, drafts="logits" if "drafts" in what else "guess")

    def tensors(x):
        if what == "place":
            return [x.lens, x.asked, x.held, x.stack, x.free, x.got["block_table"], *x.groups]
        if what == "release":
            return [x.keep, x.held, x.free, x.table, x.got["free_pages"]]
        return [x.logits, x.tokens, x.u, x.v] + ([x.draft] if x.draft is not None else [])

    call = getattr(dec, what.split()[0])
    x = make(0)
    call(x.c)                                                # (the workspace)
    x = make(1)
    graph = capture(lambda: call(x.c))
    for seed in (2, 3, 4, 5):
        y = make(seed)
        for a, b in zip(tensors(x), tensors(y)):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if what in ("place", "release"):
            x.want = y.want
        else:
            x.host = y.host
            x.exact = dec.settings == {}
        x.check((what, seed))


def test_calls_at_once(dec):
    """Two decoders on two streams, each with its own workspace, many calls each without a wait between them."""
    other = context(**dec.settings)
    try:
        runs = []
        for d, s, seed in ((dec, torch.cuda.Stream(), 1), (other, torch.cuda.Stream(), 2)):
            lens, asked, held, table, stack, free, groups = batch(seed, 1200, group=8, prefix=1)
            place = Placing(lens, asked, held, table, stack, free, int(asked.sum()), groups)
            v = [drafting(10 * seed + i, [4, 2, 5], 20000, drafts=kind) for i, kind in enumerate(("logits", "guess"))]
            runs.append((d, s, place, v))
        torch.cuda.synchronize()
        for _ in range(20):
            for d, s, place, v in runs:
                d.place(place.c, stream=s)
                for x in v:
                    d.verify(x.c, stream=s)
        torch.cuda.synchronize()
        for d, _, place, v in runs:
            place.check()
            for x in v:
                x.exact = dec.settings == {}
                x.check()
    finally:
        other.close()


def test_the_attention_reads_what_was_placed(dec):
    """A cache filled through places alone, against one whose table was made on the host: the same attention."""
    lens = [40, 3, 77, 16]
    host = Cache(lens, 2, 64)
    n = len(lens)
    table = torch.full_like(host.table_dev, -1)
    zero = ints([0] * n)
    held, cu, after, count = ints([0] * n), ints([0] * (n + 1)), ints([0] * n), ints([host.pages])
    # the stack gives the pages of the host's rows, sequence by sequence
    order = [int(p) for row, L in zip(host.table.tolist(), lens) for p in row[:su.pages_of(L)]]
    rest = [p for p in range(host.pages) if p not in order]
    dec.place(ra.place_from_tensors(zero, ints(lens), held, table, ints(rest + order[::-1]), count, cu, after, held, count))
    torch.cuda.synchronize()
    for b, L in enumerate(lens):
        assert table[b, :su.pages_of(L)].tolist() == host.table[b, :su.pages_of(L)].tolist()
    q = torch.randn((n, 4, 64), device=DEV).to(torch.bfloat16)
    outs = []
    for t in (host.table_dev, table):
        out, lse = torch.empty_like(q), torch.empty((n, 4), device=DEV)
        dec.extend(ra.extend_from_tensors(q, host.k, host.v, ints(range(n + 1)), 1, t, after, out, lse, 0.125))
        outs.append((out, lse))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
