"""How the work of the attention of chunks is divided: batches of many sequences under a page table that is wider than their
lengths need, so that no item counts as short from the start; items that are left whole, in the order of their lengths, items
that many workgroups share, and batches larger than what the search keeps on chip.  Against the 64-bit reference."""
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, Cache, Extension

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def batch(lens, chunks, Hq, Hkv, D, kv, wide):
    cache = Cache(lens, Hkv, D, kv)
    cache.table = torch.nn.functional.pad(cache.table, (0, wide), value=-1)
    cache.table_dev = cache.table.to(DEV)
    return Extension(cache, chunks, Hq)


def run(dec, what, *args):
    print("case", what, args[2:], flush=True)
    x = batch(*args)
    dec.extend(x.c)
    x.check(what)
    first = x.out.clone()
    x.out.fill_(float("nan"))
    dec.extend(x.c)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), x.out.view(torch.int16))


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,B,most", [
    (8, 8, 128, 135, 2),       # up to 32 rows
    (3, 3, 128, 350, 3),       # a number of kv heads that shares no factor with the dies
    (12, 6, 64, 264, 12),
    (32, 8, 128, 131, 9),      # up to 64 rows
    (16, 8, 128, 133, 40),     # blocks of 128 rows
    (4, 4, 64, 390, 70),
    (2, 1, 128, 512, 150),     # all sequences that the search keeps, and several blocks of some
])
def test_items_left_whole(dec, Hq, Hkv, D, B, most, kv):
    """More than twice as many items as workgroups are resident, none much longer than the others; some have no token."""
    chunks = [(1 + b % 2) * (b % 11 != 3) for b in range(B)]
    chunks[B // 2] = most
    lens = [n + (29 * b) % 90 for b, n in enumerate(chunks)]
    run(dec, "whole", lens, chunks, Hq, Hkv, D, kv, 420)


@pytest.mark.parametrize("Hq,Hkv,D,most", [(8, 8, 128, 2), (16, 8, 128, 40)])
def test_one_long_sequence_among_many(dec, Hq, Hkv, D, most):
    """As many items, one sequence far longer than the rest: its items are shared."""
    B = 132
    chunks = [1 + b % 2 for b in range(B)]
    chunks[77] = most
    lens = [n + b % 13 for b, n in enumerate(chunks)]
    lens[77] = 7900
    run(dec, "one long", lens, chunks, Hq, Hkv, D, "bf16", 0)


@pytest.mark.parametrize("B,most", [(70, 2), (70, 80), (513, 2), (700, 90), (4200, 2), (4160, 70)])
def test_batches_of_every_size(dec, B, most):
    """Batches that a wave's lanes, the search's memory and its chunks do not hold at once, with items that are shared."""
    chunks = [int(b % 5 != 2) for b in range(B)]
    chunks[B // 3], chunks[B - 1] = most, most
    lens = [n + b % 19 for b, n in enumerate(chunks)]
    lens[5], lens[B // 3], lens[B - 2] = 5900, 6100, 600
    run(dec, "size", lens, chunks, 1, 1, 64, "bf16", 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,chunk,length", [(128, 4, 2, 14000), (64, 2, 40, 14000), (128, 1, 70, 4500), (64, 1, 100, 5000)])
def test_an_item_of_many_parts(dec, D, Hq, chunk, length, kv):
    """Items of a dozen parts and more, beside one that is whole."""
    run(dec, "parts", [length, 33], [chunk, 1], Hq, 1, D, kv, 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("B", [9, 270])
@pytest.mark.parametrize("Hq,most,wide", [(4, 5, 0), (4, 5, 76), (4, 5, 100), (4, 12, 40), (4, 40, 16), (4, 40, 90)])
def test_items_that_are_short_from_the_start(dec, B, Hq, most, wide, kv):
    """Page tables on either side of the width up to which a workgroup takes an item without looking at the others."""
    chunks = [(1 + (b * 7) % most) * (b % 5 != 1) for b in range(B)]
    lens = [n + (17 * b) % 40 for b, n in enumerate(chunks)]
    run(dec, "short", lens, chunks, Hq, 1, 64, kv, wide)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,singles,pieces,deep", [
    (8, 1, 128, 1, [50], 40),                    # hardly any work: a span or two for either line
    (28, 4, 128, 12, [61, 0, 90], 700),
    (16, 2, 64, 20, [130], 900),
    (4, 4, 64, 30, [200, 150], 300),             # one head for each kv head
    (32, 1, 128, 9, [33], 1100),                 # a token's heads are all the rows that are few
])
def test_single_tokens_beside_pieces(dec, Hq, Hkv, D, singles, pieces, deep, kv):
    """Steps of most sequences and pieces of some, which are worked on apart; contexts of every length, also none."""
    chunks = [1] * singles + pieces + [1, 2, 1, 1, 1]
    lens = [n + (97 * b) % deep for b, n in enumerate(chunks)]
    lens[0] = 1
    run(dec, "beside", lens, chunks, Hq, Hkv, D, kv, 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunks", [[1, 2, 1], [70, 64], [3]])
def test_one_of_two_kinds_is_missing(dec, chunks, kv):
    """A bound that promises long chunks, over short ones alone or long ones alone."""
    x = Extension(Cache([800 + n for n in chunks], 2, 128, kv), chunks, 8, bound=600)
    dec.extend(x.c)
    x.check("missing")


@pytest.mark.parametrize("at", [0, 60, 129])
def test_later_tokens_have_no_part_beside_pieces(dec, at):
    """A NaN in one sequence's pages stays with the tokens of that sequence that see it."""
    chunks = [1, 1, 130, 2, 1, 1, 1, 1]
    cache = Cache([n + 100 for n in chunks], 2, 128)
    clean = Extension(cache, chunks, 8)
    dec.extend(clean.c)
    clean.check()
    cache.v[int(cache.table[2, (100 + at) // 16]), :, (100 + at) % 16, 5:9] = float("nan")
    x = Extension(cache, chunks, 8)
    dec.extend(x.c)
    torch.cuda.synchronize()
    spoilt = torch.isnan(x.out).any(-1).any(-1)
    assert spoilt.tolist() == [2 + at <= t < 132 for t in range(sum(chunks))]
