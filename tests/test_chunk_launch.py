"""Which way the batches of the attention's GPU tests go.  Without a workspace every item has a workgroup from the start; else the
workspace's size tells how many spans share the work, and the rest of the rule, which the device applies to the lengths, is
written out here.  For 256 compute units."""
import pytest

import paper_2507_01663_amd as ra
import test_gpu_extend_whole as whole
import test_gpu_extend_work as work

PAGE, ROWS = 16, 128


def size(lens, chunks, Hq, Hkv, D, wide=0, kv=ra.RA_KV_BF16):
    p = ra.ra_extend()
    p.num_seqs, p.total_tokens, p.max_chunk_len = len(chunks), sum(chunks), max(chunks)
    p.Hq, p.Hkv, p.D, p.page_size, p.num_pages, p.kv_dtype = Hq, Hkv, D, PAGE, 1 << 20, kv
    p.max_pages_per_seq = max(1, max((x + PAGE - 1) // PAGE for x in lens)) + wide
    return ra.rollout_attn_extend_workspace_size(None, p)


def spans(n, D):
    """Two slots of 128 rows for each, with their statistics, and two descriptors of 16 bytes."""
    each = 2 * ROWS * (4 * D + 8) + 32
    assert n // each % 8 == 0 and n % each < 3 * 256
    return n // each


def params(test):
    """The arguments of a test's parametrize marks, by name."""
    return {m.args[0]: m.args[1] for m in test.pytestmark if m.name == "parametrize"}


def left_whole(lens, chunks, Hq, Hkv, D, wide):
    """Are there twice as many items as spans, and is none longer than a span?"""
    n, G, most = spans(size(lens, chunks, Hq, Hkv, D, wide), D), Hq // Hkv, max(chunks)
    two = most * G > 64 and 4 * sum(chunks) <= len(chunks) * most
    total = items = longest = 0
    for c, L in zip(chunks, lens):
        if c:
            rows = 32 if two and c * G <= 32 else most * G
            fixed, stages = 8 if rows > 64 and not two else 4, (L - c // 2 + 48) >> 5
            cost = fixed + 1 + (stages if rows > 64 else stages * (14 if rows > 32 else 9) >> 5)
            blocks = -(-c * G // ROWS)
            total, items, longest = total + Hkv * blocks * cost, items + Hkv * blocks, max(longest, cost)
    least = 6 + (8 if most * G > 64 and not two else 4)
    share = total // (n if total >= least * n else max(1, total // least))
    return items >= 2 * n and longest <= share


def test_batches_of_whole_items():
    for Hq, Hkv, D, B, most in whole.SHAPES:
        chunks, lens = whole.batch(B, most)
        assert left_whole(lens, chunks, Hq, Hkv, D, whole.WIDE), (Hq, Hkv, D, B, most)
    for Hq, Hkv, D, B in whole.LONG:
        chunks, lens = whole.long_chunks(B)
        assert left_whole(lens, chunks, Hq, Hkv, D, whole.WIDE), (Hq, Hkv, D, B)


def test_shared_items_have_a_workspace():
    for D, Hq, chunk, length in params(work.test_an_item_of_many_parts)["D,Hq,chunk,length"]:
        assert spans(size([length, 33], [chunk, 1], Hq, 1, D), D) >= 16
    for B, most in params(work.test_batches_of_every_size)["B,most"]:
        chunks = [int(b % 5 != 2) for b in range(B)]
        chunks[B // 3], chunks[B - 1] = most, most
        assert size([6100] * B, chunks, 1, 1, 64) > 0


@pytest.mark.parametrize("B", params(work.test_items_that_are_short_from_the_start)["B"])
def test_page_tables_on_either_side_of_the_width(B):
    """Of the tables that are said to be so, some leave every item short and some do not."""
    ways = []
    for Hq, most, wide in params(work.test_items_that_are_short_from_the_start)["Hq,most,wide"]:
        chunks = [(1 + (b * 7) % most) * (b % 5 != 1) for b in range(B)]
        lens = [n + (17 * b) % 40 for b, n in enumerate(chunks)]
        ways.append(size(lens, chunks, Hq, 1, 64, wide) == 0)
    assert True in ways and False in ways, ways


def test_the_width_decides():
    """One chunk: no workspace under a narrow table, one under a wide table, and a change at one width."""
    for Hq, Hkv, D, chunk in ((4, 2, 64, 17), (8, 2, 128, 5), (8, 2, 128, 100)):
        ways = [size([16], [chunk], Hq, Hkv, D, wide) == 0 for wide in range(0, 400)]
        assert ways[0] and not ways[-1] and ways == sorted(ways, reverse=True)
