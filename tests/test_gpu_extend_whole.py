"""Batches of so many items of about one length that a workgroup takes each of them whole, in the order of their lengths, under a page
table with room for long ones: for every kind of kernel, pool type and number of kv heads, with sequences that have no token.
Against the 64-bit reference.  (That the sizes do so for 256 compute units is asserted on the host.)"""
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, Cache, Extension

pytestmark = pytest.mark.gpu

WIDE = 420
# (query heads, kv heads, D, sequences, the longest chunk)
SHAPES = [
    (8, 8, 128, 150, 2),       # up to 32 rows
    (3, 3, 128, 390, 3),       # a number of kv heads that shares no factor with the dies
    (12, 6, 64, 290, 12),
    (32, 8, 128, 150, 9),      # up to 64 rows
    (64, 16, 64, 110, 16),
    (16, 8, 128, 150, 40),     # blocks of 128 rows, most sequences far shorter: two kinds beside each other
    (4, 4, 64, 440, 70),
    (8, 4, 128, 300, 40),
]


def batch(B, most):
    chunks = [(1 + b % 2) * (b % 11 != 3) for b in range(B)]
    chunks[B // 2] = most
    return chunks, [n + (29 * b) % 90 for b, n in enumerate(chunks)]


def long_chunks(B):
    """Chunks of one or two blocks of 128 rows of two heads, none far shorter than the longest."""
    chunks = [33 + (17 * b) % 60 for b in range(B)]
    return chunks, [n + (29 * b) % 50 for b, n in enumerate(chunks)]


LONG = [(8, 4, 64, 290), (16, 8, 128, 100)]


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def run(dec, chunks, lens, Hq, Hkv, D, kv):
    cache = Cache(lens, Hkv, D, kv)
    cache.table = torch.nn.functional.pad(cache.table, (0, WIDE), value=-1)
    cache.table_dev = cache.table.to(DEV)
    x = Extension(cache, chunks, Hq)
    dec.extend(x.c)
    x.check("whole")
    first = x.out.clone()
    x.out.fill_(float("nan"))
    dec.extend(x.c)
    torch.cuda.synchronize()
    assert torch.equal(first.view(torch.int16), x.out.view(torch.int16))


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,B,most", SHAPES)
def test_many_items(dec, Hq, Hkv, D, B, most, kv):
    print("case", Hq, Hkv, D, B, most, kv, flush=True)
    run(dec, *batch(B, most), Hq, Hkv, D, kv)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,B", LONG)
def test_many_items_of_several_blocks(dec, Hq, Hkv, D, B, kv):
    print("case", Hq, Hkv, D, B, kv, flush=True)
    run(dec, *long_chunks(B), Hq, Hkv, D, kv)
