"""Chunks longer than the bound that the call gives: the tokens before the bound have the results that the definition gives them
(what is at or past it may be left out).  Against the 64-bit reference."""
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import U, Cache, Extension, attention

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def check(x, bound, what):
    """As Extension.check, of every chunk's tokens before the bound."""
    torch.cuda.synchronize()
    out, lse, t = x.out.double().cpu(), x.lse.double().cpu(), 0
    for b, n in enumerate(x.chunks):
        m, L = min(n, bound), x.totals[b]
        ref, rlse, mag = attention(x.q_host[t:t + m].double(), x.cache.values("k", b, L), x.cache.values("v", b, L), L - n, x.scale)
        err = (out[t:t + m] - ref).abs() - 1.1 * U * (ref.abs() + mag) - 1e-6
        assert m == 0 or err.max() <= 0, (what, b, float(err.max()))
        assert torch.equal(torch.isneginf(rlse), torch.isneginf(lse[t:t + m])), (what, b)
        fine = torch.isfinite(rlse)
        assert not fine.any() or (rlse - lse[t:t + m])[fine].abs().max() <= 1e-4, (what, b)
        t += n


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,chunks,lens,bound,wide", [
    (8, 2, 128, [9, 1, 4], [90, 17, 4], 3, 0),                   # up to 32 rows
    (8, 2, 64, [40, 2, 17], [95, 60, 33], 16, 0),                # up to 64
    (8, 2, 128, [90, 33, 70], [200, 65, 70], 64, 0),             # blocks of rows, a chunk without a context
    (8, 2, 128, [9, 1, 4], [900, 17, 4], 3, 400),                # the same under a wide page table: shared items
    (4, 1, 64, [90, 33, 70], [1200, 65, 70], 64, 400),
    (8, 1, 128, [1, 1, 1, 200, 1, 2, 1, 1], [5, 40, 90, 430, 1, 77, 600, 31], 110, 400),     # short ones beside long ones
    (8, 2, 128, [1, 2, 5, 0], [33, 34, 70, 9], 1, 0),            # a bound of one that is not a decode step
])
def test_chunks_longer_than_the_bound(dec, Hq, Hkv, D, chunks, lens, bound, wide, kv):
    print("case", Hq, Hkv, D, chunks, lens, bound, wide, kv, flush=True)
    cache = Cache(lens, Hkv, D, kv)
    cache.table = torch.nn.functional.pad(cache.table, (0, wide), value=-1)
    cache.table_dev = cache.table.to(cache.table_dev.device)
    x = Extension(cache, chunks, Hq, bound=bound)
    dec.extend(x.c)
    check(x, bound, "bound")


def test_many_items_left_whole_and_longer_than_the_bound(dec):
    B = 132
    chunks = [1 + b % 3 for b in range(B)]
    lens = [n + (29 * b) % 90 for b, n in enumerate(chunks)]
    cache = Cache(lens, 8, 128)
    cache.table = torch.nn.functional.pad(cache.table, (0, 420), value=-1)
    cache.table_dev = cache.table.to(cache.table_dev.device)
    x = Extension(cache, chunks, 16, bound=2)
    dec.extend(x.c)
    check(x, 2, "whole")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_fewer_keys_than_tokens_and_a_bound(dec, kv):
    """Lengths below the chunk's, and below what the bound leaves of it."""
    cache = Cache([80, 80, 80, 80], 2, 128, kv)
    for bound, chunks, totals in ((4, [9, 9, 9, 9], [9, 7, 3, 0]), (40, [70, 60, 65, 50], [35, 80, 20, 0])):
        x = Extension(cache, chunks, 8, totals=totals, bound=bound)
        dec.extend(x.c)
        check(x, bound, "short")
