"""Places of new tokens and pages back to the stack, on the GPU, against the plain forms.  All whole numbers: equal."""
import numpy as np
import pytest
import torch

import paper_2507_01663_amd as ra
from step_util import DEV, PAGE, Placing, Releasing, batch, ints, pages_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def run(dec, x, what=""):
    (dec.place if isinstance(x, Placing) else dec.release)(x.c)
    return x.check(what)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 300, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("slack", [1.0, 0.7])
def test_batches(dec, n, slack):
    """Enough pages, or too few; room for all tokens, some more, or fewer; in place or not; ragged, with sequences that ask for none."""
    for seed, (group, prefix) in enumerate([(0, 0), (4, 3), (8, 1)]):
        lens, asked, held, table, stack, free, groups = batch(100 * n + seed, n, group=group, prefix=prefix, slack=slack)
        total = int(asked.sum())
        for room in (total, total + 700, max(0, total - 50)):
            for alias in (False, True):
                print("case", n, slack, group, room, alias, flush=True)
                run(dec, Placing(lens, asked, held, table, stack, free, room, groups, alias))
        back = Releasing(np.maximum(0, lens - np.arange(n) % 40), held, table, stack, free, groups, alias=seed == 1)
        run(dec, back)


@pytest.mark.parametrize("n", [64, 1023, 1024, 1025, 2048, 2500])
@pytest.mark.parametrize("slack", [1.0, 0.7])
def test_steps_of_few_tokens(dec, n, slack):
    """At most four new tokens a sequence and 1024 in a tile of 1024 sequences, which sequences place themselves: one for all, one for some, up to
    four for some; and tiles of that kind before and behind one with a turn in it, or with more tokens than threads, or with a turn that
    is not served.  With groups, too few pages, room for all, more or fewer tokens, in place or not."""
    r = np.random.default_rng(n)
    one, few = np.ones(n, dtype=np.int64), np.where(r.random(n) < 0.35, r.integers(1, 5, n), 0)
    first, last, many, huge = few.copy(), few.copy(), few.copy(), few.copy()
    first[min(5, n - 1)], last[n - 1], many[-(n // 5):] = 60, 61, 4
    huge[[0, n // 2, n - 1]] = 100000                        # (more than a row has room for)
    for seed, (group, prefix) in enumerate([(0, 0), (8, 2)]):
        for name, asked in (("one", one), ("few", few), ("first", first), ("last", last), ("many", many), ("huge", huge)):
            lens, _, held, table, stack, _, groups = batch(10 * n + seed, n, new=64, group=group, prefix=prefix, slack=1.0)
            shared = [prefix if group and groups[0][b] >= 0 else 0 for b in range(n)]
            need = sum(max(0, pages_of(int(a + k)) - max(int(h), s)) for a, k, h, s in zip(lens, asked, held, shared) if 0 < k < 100)
            total = int(asked[asked < 100].sum())
            for room in (total, min(4096, total + 700), total // 2):
                for alias in (False, True):
                    print("case", n, slack, group, name, room, alias, flush=True)
                    assert room <= 4096
                    run(dec, Placing(lens, asked, held, table, stack, int(need * slack), room, groups, alias), (name, group, room, alias))


@pytest.mark.parametrize("tokens", [1, 15, 16, 17, 4095, 4096, 5000, 70000])
def test_one_sequence(dec, tokens):
    for held_tokens in (0, 1, 15, 16, 31):
        L, h = held_tokens, pages_of(held_tokens)
        M = pages_of(L + tokens) + 1
        table = np.full((1, M), -1, dtype=np.int32)
        table[0, :h] = [2000000 + i for i in range(h)]
        stack = np.random.default_rng(tokens).permutation(M + 3)
        for free in (pages_of(L + tokens) - h, pages_of(L + tokens) - h - 1, len(stack)):
            if free >= 0:
                run(dec, Placing([L], [tokens], [h], table, stack, free, tokens))


def test_long_prompts_of_many_sequences(dec):
    """More tokens than one workgroup is given, and pages given back that are as many."""
    lens, asked, held, table, stack, free, groups = batch(5, 1100, most=900, new=700)
    run(dec, Placing(lens, asked, held, table, stack, free, int(asked.sum()) + 5000))
    run(dec, Placing(lens, asked, held, table, stack, free, int(asked.sum()), alias=True))
    stack = np.concatenate([stack, np.full(int(held.sum()), -5)])
    for alias in (False, True):
        run(dec, Releasing(np.zeros(1100), held, table, stack, free, alias=alias))
    run(dec, Releasing(np.where(np.arange(1100) % 3, lens, lens // 2), held, table, stack, free))


def test_what_is_not_considered(dec):
    """Negative lengths and counts, rows that do not hold their tokens, more than a row has room for: left as they are, and in nobody's
    way."""
    big = 2 ** 31 - 1
    lens = [5, -1, 40, 3, 16, 0, big, 0, 7, 10]
    asked = [0, 4, 4, -3, 4, big, 1, 81, 9, 20]
    held = [1, 1, 2, 1, -1, 0, 1, 0, 6, 1]
    table = np.arange(50, dtype=np.int32).reshape(10, 5)
    stack = np.arange(100, 120)
    for free in (20, 3, 1, 0, -4, 25, 10 ** 9):
        run(dec, Placing(lens, asked, held, table, stack, free, 60))
        run(dec, Releasing(lens, held, table, stack, free))


def test_groups(dec):
    """New members of a group take its pages into their rows, in part where they hold some; unknown groups count as none; a prefix that
    the row has no room for, or that shrinks, is not considered or shares none."""
    table = np.arange(40, dtype=np.int32).reshape(8, 5)
    groups = ([0, 0, 1, -1, 5, -7, 2, 3], [0, 3, 3, 9, 7], [90, 91, 92, 93, 94, 95, 96, 97, 98])
    lens, asked, held = [48, 48, 5, 4, 4, 4, 16, 3], [3, 17, 4, 5, 30, 2, 4, 4], [0, 2, 1, 1, 1, 1, 1, 1]
    for free in (6, 2):
        run(dec, Placing(lens, asked, held, table, np.arange(200, 206), free, 100, groups))
        run(dec, Releasing([0, 20, 5, 0, 4, 100, 16, 3], [4, 5, 1, 2, 3, 1, 1, 5], table, np.arange(200, 220), free, groups))


def test_nothing_to_place(dec):
    none = np.zeros((0, 4), dtype=np.int32)
    run(dec, Placing([], [], [], none, [3, 4, 5], 2, 0))
    run(dec, Placing([], [], [], none, [3, 4, 5], 2, 5))
    run(dec, Releasing([], [], none, [3, 4, 5], 2))
    run(dec, Placing([4, 5], [0, 0], [1, 1], np.zeros((2, 4), dtype=np.int32), [], 0, 9))
    run(dec, Placing([4, 5], [3, 20], [1, 1], np.zeros((2, 4), dtype=np.int32), [], 0, 9))
    run(dec, Placing([0, 0], [3, 20], [0, 0], np.zeros((2, 0), dtype=np.int32), [1, 2], 2, 9))
    run(dec, Releasing([0, 0], [0, 0], np.zeros((2, 0), dtype=np.int32), [1, 2], 2))


def test_a_full_stack_takes_no_more(dec):
    table = np.arange(12, dtype=np.int32).reshape(3, 4)
    run(dec, Releasing([0, 0, 0], [3, 4, 2], table, np.arange(20, 26), 1))


def test_outputs_that_are_not_wanted(dec):
    lens, asked, held, table, stack, free, groups = batch(9, 200)
    x = Placing(lens, asked, held, table, stack, free, int(asked.sum()), tokens=False)
    run(dec, x)
    x = Placing(lens, asked, held, table, stack, free, int(asked.sum()))
    x.c.positions = x.c.seqs = None
    for name in ("positions", "seqs"):
        assert (x.got.pop(name) == -77).all()
    run(dec, x)


def test_twice_and_on_another_stream(dec):
    lens, asked, held, table, stack, free, groups = batch(11, 1500, group=8, prefix=2)
    x = Placing(lens, asked, held, table, stack, free, int(asked.sum()), groups)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    dec.place(x.c, stream=s)
    dec.place(x.c, stream=s)                                 # (the same inputs: the same places)
    x.check()


def test_grow_and_shrink_for_many_steps(dec):
    """In place over many steps, sequences that end and begin again: no page is ever in two rows, and all of them come back."""
    r = np.random.default_rng(0)
    n, M, pages = 50, 20, 400
    lens, held, free = (torch.zeros(k, dtype=torch.int32, device=DEV) for k in (n, n, 1))
    stack = ints(r.permutation(pages))
    free.fill_(pages)
    table = torch.full((n, M), -1, dtype=torch.int32, device=DEV)
    cu, keep, asked = ints([0] * (n + 1)), ints([0] * n), ints([0] * n)
    room = 2000
    grow = ra.place_from_tensors(lens, asked, held, table, stack, free, cu, lens, held, free, total_tokens=room)
    shrink = ra.release_from_tensors(keep, held, table, stack, free, held, free)
    for step in range(60):
        asked.copy_(ints(r.integers(0, 40, n)))
        was = lens.clone()
        dec.place(grow)
        assert int(cu[-1]) == int((lens - was).sum())
        keep.copy_(torch.where(ints(r.random(n) < 0.15) > 0, 0, (lens - ints(r.integers(0, 5, n))).clamp(min=0)))
        if step % 3 == 0:
            dec.release(shrink)
            lens.copy_(torch.minimum(lens, keep))
        rows = [table[b, :int(held[b])].tolist() for b in range(n)]
        used = sorted(p for row in rows for p in row)
        assert sorted(used + stack[:int(free)].tolist()) == list(range(pages))
        assert all(len(row) * PAGE >= int(L) for row, L in zip(rows, lens.tolist()))
    keep.zero_()
    dec.release(shrink)
    assert int(free) == pages and sorted(stack.tolist()) == list(range(pages))
