"""Appends of so many rows that a wave takes four passes, for both head dims and pool types, with head counts that leave the last
pass partly empty and ones that fill it.  Rows of sampled sequences against the 64-bit reference; the rest against the same
sequences appended alone, which a pass for each wave does."""
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, PAGE, cu_of, ints, normal, rotated
from test_gpu_rotate import close, packed, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def passes(T, rows, D):
    """Passes of a wave that the rows of T tokens need: 64 lanes, D / 16 of them to a row."""
    slots = 64 // (D // 16)
    per = 1
    while per < rows and per < slots:
        per *= 2
    return -(-T // (slots // per)) * -(-rows // per)


# (query heads, kv heads, D, tokens)
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,T", [(37, 1, 64, 3100), (32, 2, 64, 4500), (41, 3, 128, 1700), (28, 4, 128, 2300), (5, 1, 64, 20000), (64, 8, 128, 1100)])
def test_four_passes(dec, Hq, Hkv, D, T, kv):
    rows = Hq if kv == "e4m3" else Hq + 2 * Hkv
    assert passes(T, rows, D) > 32 * torch.cuda.get_device_properties(0).multi_processor_count
    g = torch.Generator().manual_seed(T)
    chunks, left = [], T
    while left:
        chunks.append(min(left, int(torch.randint(0, 400, (1,), generator=g))))
        left -= chunks[-1]
    B = len(chunks)
    before = torch.randint(0, 60, (B,), generator=g).tolist()
    pages = [(a + n + PAGE - 1) // PAGE for a, n in zip(before, chunks)]
    table = torch.full((B, max(pages)), -1, dtype=torch.int32)
    ids, at = torch.randperm(sum(pages), generator=g).to(torch.int32), 0
    for b, n in enumerate(pages):
        table[b, :n] = ids[at:at + n]
        at += n
    x, q, k, v = packed(T, Hq, Hkv, D, 11)
    qw, kw = weights(D, 4)
    rope = ra.rope_table(600, D, 1e4, "cpu")
    turn = [t.to(DEV) for t in (rope, qw, kw)]
    table_dev, cu, lens = table.to(DEV), cu_of(chunks), ints(before)

    def pools():
        """What is stored before: some pages' scales are kept, the others' renewed."""
        h = torch.Generator().manual_seed(7)
        shape = (sum(pages), Hkv, PAGE, D)
        if kv == "bf16":
            return [torch.randn(shape, generator=h).to(torch.bfloat16).to(DEV) for _ in "kv"] + [None, None]
        codes = [torch.randint(0, 0x7f, shape, generator=h, dtype=torch.uint8).to(DEV) for _ in "kv"]
        return codes + [(0.02 * torch.rand(shape[:2], generator=h)).to(DEV) for _ in "kv"]

    def append(of, part, b0, b1):
        t0, t1 = sum(chunks[:b0]), sum(chunks[:b1])
        cu_part, most = cu_of(chunks[b0:b1]), max(chunks[b0:b1])
        out = part[t0:t1]
        lens_part, table_part = lens[b0:b1].contiguous(), table_dev[b0:b1].contiguous()
        dec.append_chunk(ra.append_chunk_from_tensors(k[t0:t1], v[t0:t1], cu_part, most, table_part, lens_part, *of[:2], *of[2:], q=q[t0:t1], q_out=out,
                                                      rope=turn[0], q_weight=turn[1], k_weight=turn[2]))
        torch.cuda.synchronize()

    whole, apart = pools(), pools()
    q_whole, q_apart = (torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in "ab")
    print("case", Hq, Hkv, D, T, kv, "sequences", B, flush=True)
    append(whole, q_whole, 0, B)
    for b in range(B):
        if chunks[b]:
            append(apart, q_apart, b, b + 1)
    assert torch.equal(q_whole.view(torch.int16), q_apart.view(torch.int16))
    for a, b in zip(whole, apart):
        assert a is None or torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    place = torch.cat([torch.arange(a, a + n) for a, n in zip(before, chunks)])
    some = torch.cat([torch.arange(0, 30), torch.arange(T // 2, T // 2 + 30), torch.arange(T - 30, T)])
    close(q_whole[some], rotated(q[some].double().cpu(), qw, place[some], rope))
    if kv == "bf16":
        owner = torch.repeat_interleave(torch.arange(B), torch.tensor(chunks))
        page = table[owner[some], place[some] // PAGE].long()
        close(whole[0][page.to(DEV), :, (place[some] % PAGE).to(DEV)], rotated(k[some].double().cpu(), kw, place[some], rope))
        assert torch.equal(whole[1][page.to(DEV), :, (place[some] % PAGE).to(DEV)].view(torch.int16), v[some].contiguous().view(torch.int16))
