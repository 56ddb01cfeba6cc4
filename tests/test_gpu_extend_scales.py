"""e4m3 pages that a token does not see: whatever their scales are has no part in the token's result.  A page's scale becomes
infinite when an infinite value is appended; a NaN is one that nothing appended."""
import numpy as np
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, PAGE, Cache, Extension, cu_of, ints, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def bits(x):
    return x.view(torch.int16 if x.element_size() == 2 else torch.int32).cpu()


# (query heads, kv heads, D, new tokens, length): up to 32 rows, up to 64, blocks of rows, an item that workgroups share
SHAPES = [(8, 2, 128, 8, 148), (8, 2, 64, 8, 148), (8, 2, 128, 16, 152), (8, 2, 64, 15, 151), (8, 2, 128, 70, 150), (8, 2, 64, 70, 150),
          (2, 1, 128, 40, 71), (32, 1, 128, 5, 66), (4, 1, 128, 6, 4036), (4, 1, 64, 50, 3030)]


def later_pages(chunk, L):
    """The pages that some of the chunk's tokens do not see and others do."""
    return [p for p in range((L + PAGE - 1) // PAGE) if p * PAGE > L - chunk]


@pytest.mark.parametrize("which", ["ks", "vs"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("Hq,Hkv,D,chunk,L", SHAPES)
def test_scales_of_later_pages(dec, Hq, Hkv, D, chunk, L, bad, which):
    cache = Cache([L], Hkv, D, "e4m3")
    clean = Extension(cache, [chunk], Hq)
    dec.extend(clean.c)
    clean.check("clean")
    pages = later_pages(chunk, L)
    assert pages
    for p in pages:
        print("case", Hq, Hkv, D, chunk, L, which, bad, "page", p, flush=True)
        scale = getattr(cache, which)
        was = scale.clone()
        scale[int(cache.table[0, p])] = bad
        x = Extension(cache, [chunk], Hq)
        dec.extend(x.c)
        torch.cuda.synchronize()
        scale.copy_(was)
        before = p * PAGE - (L - chunk)              # tokens that do not see the page
        assert torch.equal(bits(x.out[:before]), bits(clean.out[:before])) and torch.equal(bits(x.lse[:before]), bits(clean.lse[:before]))
        if which == "vs":
            assert not torch.isfinite(x.out[before:]).any() and torch.equal(bits(x.lse), bits(clean.lse))
        elif bad != bad:
            assert torch.isnan(x.out[before:]).all() and torch.isnan(x.lse[before:]).all()


@pytest.mark.parametrize("which", ["ks", "vs"])
@pytest.mark.parametrize("chunks", [[1, 1, 130, 2, 1, 1, 1, 1], [1, 3, 7, 2, 1, 1], [3, 0, 90, 70, 1]])
def test_scales_of_later_pages_in_a_batch(dec, chunks, which):
    """A step of short and long chunks: one page of one sequence, in turn."""
    lens = [n + 41 + 3 * b for b, n in enumerate(chunks)]
    cache = Cache(lens, 2, 128, "e4m3")
    clean = Extension(cache, chunks, 8)
    dec.extend(clean.c)
    clean.check("clean")
    scale = getattr(cache, which)
    was = scale.clone()
    start = 0
    for b, n in enumerate(chunks):
        for p in later_pages(n, lens[b]):
            scale[int(cache.table[b, p])] = float("inf" if which == "vs" else "nan")
            x = Extension(cache, chunks, 8)
            dec.extend(x.c)
            torch.cuda.synchronize()
            scale.copy_(was)
            first = start + p * PAGE - (lens[b] - n)
            rest = [t for t in range(sum(chunks)) if not first <= t < start + n]
            assert torch.equal(bits(x.out[rest]), bits(clean.out[rest])) and torch.equal(bits(x.lse[rest]), bits(clean.lse[rest])), (b, p)
            assert not torch.isfinite(x.out[first:start + n]).any(), (b, p)
        start += n


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("Hq,n,before,at", [(8, 32, 0, 20), (2, 32, 0, 20), (8, 8, 28, 34), (8, 90, 20, 52)])
def test_an_infinite_value_on_its_way_through_the_cache(dec, Hq, n, before, at, which, value):
    """append_chunk, then extend: a value of token `at` that is infinite or NaN changes nothing for tokens that do not see its page."""
    Hkv, D = 2, 128
    L = before + n
    got = []
    for odd in (False, True):
        cache = Cache([before], Hkv, D, "e4m3", room=n)
        k, v = normal((n, Hkv, D), 5), normal((n, Hkv, D), 6)
        (k if which == "k" else v)[at - before, :, 7] = value if odd else 0.0
        k, v, cu, lens = k.to(DEV), v.to(DEV), cu_of([n]), ints([before])
        dec.append_chunk(ra.append_chunk_from_tensors(k, v, cu, n, cache.table_dev, lens, cache.k, cache.v, cache.ks, cache.vs))
        x = Extension(cache, [n], Hq, totals=[L])
        dec.extend(x.c)
        torch.cuda.synchronize()
        got.append(x)
    clean, x = got
    clean.check("clean")
    # the tokens before the odd one's page; a NaN has no part in the scale, so that those before it in its page keep theirs too
    same = (at if value != value else at // PAGE * PAGE) - before
    assert same > 0
    assert torch.equal(bits(x.out[:same]), bits(clean.out[:same])) and torch.equal(bits(x.lse[:same]), bits(clean.lse[:same]))
    assert not torch.isfinite(x.out[at - before:, :, 7] if which == "v" else x.out[at - before:]).any()

@pytest.mark.parametrize("Hq,chunk,L", [(8, 8, 148), (8, 16, 152), (8, 70, 150)])
def test_scores_that_underflow(dec, Hq, chunk, L):
    """A page's scale times the softmax scale is below the smallest number: all scores are zero, and every key that is seen
    weighs the same."""
    cache = Cache([L], 2, 128, "e4m3")
    cache.ks.fill_(1e-20)
    x = Extension(cache, [chunk], Hq)
    x.scale = float(np.float32(1e-30))
    x.c.softmax_scale = x.scale
    dec.extend(x.c)
    x.check("underflow")
