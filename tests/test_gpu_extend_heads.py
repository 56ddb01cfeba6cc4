"""Attention of chunks where one token's query heads of a kv head fill more than a group of 32 rows: up to 128 of them."""
import pytest

import paper_2507_01663_amd as ra
from chunk_util import Cache, Extension

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,Hkv", [(33, 1), (48, 2), (64, 1), (65, 1), (71, 2), (96, 1), (127, 1), (128, 2)])
@pytest.mark.parametrize("chunks,lens", [([1, 1], [40, 17]), ([3, 1, 0, 2], [3, 50, 9, 90]), ([2, 5], [2100, 33])])
def test_many_heads_to_a_kv_head(dec, G, Hkv, D, chunks, lens, kv):
    print("case", G, Hkv, D, chunks, lens, kv, flush=True)
    x = Extension(Cache(lens, Hkv, D, kv), chunks, G * Hkv)
    dec.extend(x.c)
    x.check("heads")
