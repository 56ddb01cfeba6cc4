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
    run(dec, "whole", lens, chunks, Hq, Hkv, D, kv, 130)


@pytest.mark.parametrize("Hq,Hkv,D,most", [(8, 8, 128, 2), (16, 8, 128, 40)])
def test_one_long_sequence_among_many(dec, Hq, Hkv, D, most):
    """As many items, one sequence far longer than the rest: its items are shared."""
    B = 132
    chunks = [1 + b % 2 for b in range(B)]
    chunks[77] = most
    lens = [n + b % 13 for b, n in enumerate(chunks)]
    lens[77] = 2900
    run(dec, "one long", lens, chunks, Hq, Hkv, D, "bf16", 0)


@pytest.mark.parametrize("B,most", [(70, 2), (70, 80), (513, 2), (700, 90), (4200, 2), (4160, 70)])
def test_batches_of_every_size(dec, B, most):
    """Batches that a wave's lanes, the search's memory and its chunks do not hold at once, with items that are shared."""
    chunks = [int(b % 5 != 2) for b in range(B)]
    chunks[B // 3], chunks[B - 1] = most, most
    lens = [n + b % 19 for b, n in enumerate(chunks)]
    lens[5], lens[B // 3], lens[B - 2] = 1900, 2100, 600
    run(dec, "size", lens, chunks, 1, 1, 64, "bf16", 0)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D,Hq,chunk,length", [(128, 4, 2, 14000), (64, 2, 40, 14000), (128, 1, 70, 4500), (64, 1, 100, 5000)])
def test_an_item_of_many_parts(dec, D, Hq, chunk, length, kv):
    """Items of a dozen parts and more, beside one that is whole."""
    run(dec, "parts", [length, 33], [chunk, 1], Hq, 1, D, kv, 0)
