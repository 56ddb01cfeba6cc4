"""Attention of chunks of new tokens over the paged cache, on the GPU, against the 64-bit reference: head layouts, lengths and
masks where it can go wrong, both pool types, what a token does not see, launch shapes, streams, graphs."""
import ctypes

import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, PAGE, Cache, Extension, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def run(dec, cache, chunks, Hq, what="", **kw):
    print("case", what, "Hq", Hq, "Hkv", cache.Hkv, "D", cache.D, cache.kv, "chunks", chunks[:8], "lens", cache.lens[:8], flush=True)
    x = Extension(cache, chunks, Hq, **kw)
    dec.extend(x.c)
    return x.check(what)


HEADS = [(4, 2, 64), (7, 1, 64), (8, 8, 64), (32, 2, 64), (28, 4, 128), (5, 1, 128), (8, 8, 128), (16, 1, 128), (32, 1, 128)]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_few_rows(dec, Hq, Hkv, D, kv):
    """Chunks whose rows of a kv head fit one pass: up to 64 of them."""
    G = Hq // Hkv
    for most in sorted({max(1, 16 // G), max(1, 32 // G), 64 // G}):
        chunks = [most, 1, max(1, most - 1), min(2, most), most, min(most, 3)]
        if max(chunks) == 1:
            chunks[1] = 0                      # (one token for every sequence would be a decode step)
        lens = [most, 1 + 30, 16 * 5, 33, 16 * 20 + 1, 257]
        run(dec, Cache(lens, Hkv, D, kv, seed=most), chunks, Hq, "few %d" % most)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
def test_many_rows(dec, Hq, Hkv, D, kv):
    """Chunks of several blocks of rows, beginning and ending inside pages, stages and blocks; one with no token, one alone."""
    chunks = [65, 0, 1, 33, 97]
    lens = [65, 40, 77, 33 + 128, 97 + 31]
    run(dec, Cache(lens, Hkv, D, kv), chunks, Hq, "many")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [3, 40])
@pytest.mark.parametrize("before", [0, 1, 14, 15, 16, 17, 31, 32, 33, 63, 65])
def test_lengths_around_pages_and_stages(dec, before, chunk, kv):
    run(dec, Cache([before + chunk], 2, 128, kv, seed=before), [chunk], 8, "before %d" % before)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,Hkv,D,chunks,lens", [
    (8, 2, 128, [5], [3000]),                 # one item per kv head, shared by many workgroups
    (8, 2, 64, [4, 2], [2500, 40]),
    (8, 2, 128, [70], [2100]),
    (4, 1, 64, [130, 9], [1500, 60]),
    (16, 2, 128, [3, 1, 2, 3], [1700, 20, 900, 333]),
    (28, 4, 128, [30, 64], [900, 1500]),
])
def test_items_that_workgroups_share(dec, Hq, Hkv, D, chunks, lens, kv):
    run(dec, Cache(lens, Hkv, D, kv), chunks, Hq, "shared")


@pytest.mark.parametrize("chunks", [[2] * 70, [40] + [1] * 69, [0] * 69 + [3], [1, 0] * 150])
def test_batches_beyond_a_wave(dec, chunks):
    """More sequences than a wave looks at together; most of them without a token, or with one."""
    lens = [n + (37 * b) % 90 for b, n in enumerate(chunks)]
    run(dec, Cache(lens, 1, 64), chunks, 2, "wide")


def test_very_large_batch(dec):
    """More sequences than the lanes have chunks of."""
    chunks = [1 + (b % 7 == 0) for b in range(4200)]
    lens = [n + b % 5 for b, n in enumerate(chunks)]
    run(dec, Cache(lens, 1, 64), chunks, 1, "very wide")


def test_single_tokens_are_a_decode_step(dec):
    """One token for every sequence: the decode step's bytes."""
    for kv in ("bf16", "e4m3"):
        cache = Cache([1, 16, 17, 300, 0], 2, 128, kv)
        x = run(dec, cache, [1] * 5, 8, "single", totals=cache.lens)
        out, lse = torch.empty_like(x.out), torch.empty_like(x.lse)
        dec.decode(ra.problem_from_tensors(x.q, cache.k, cache.v, cache.table_dev, x.after, out, lse, x.scale, k_scale=cache.ks, v_scale=cache.vs))
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), x.out.view(torch.int16)) and torch.equal(lse, x.lse)
    # ... also where the decode step does not have the shape
    run(dec, Cache([5, 40, 90], 1, 64), [1, 1, 1], 32, "single, many heads")
    run(dec, Cache([5, 40, 90], 2, 64), [1, 1, 1], 4, "single, strided", q_gap=64)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["phd", "gaps"])
@pytest.mark.parametrize("chunks", [[4, 9], [60, 33]])
def test_strides(dec, layout, chunks, kv):
    run(dec, Cache([200, 95], 2, 128, kv, layout=layout), chunks, 8, layout, q_gap=72)
    run(dec, Cache([200, 95], 2, 64, kv, layout=layout), chunks, 4, layout, q_gap=8)


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunks", [[6, 3, 2], [70, 40, 9]])
def test_tokens_that_see_nothing(dec, chunks, kv):
    """Fewer tokens in the cache than in the chunk: the first ones see no key.  Empty caches and lengths out of range."""
    cache = Cache([400, 400, 400], 2, 128, kv)
    run(dec, cache, chunks, 8, "short", totals=[2, 0, 1])
    if chunks[0] > 40:
        run(dec, cache, chunks, 8, "short", totals=[37, 39, 1])
    x = Extension(cache, chunks, 8, totals=[0, 0, 400])
    x.after.copy_(torch.tensor([-5, -2 ** 31, 10 ** 6], dtype=torch.int32))     # as 0, 0 and what the table has room for
    x.totals = [0, 0, cache.table.shape[1] * PAGE]
    dec.extend(x.c)
    x.check("out of range")


@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,chunk,at", [(8, 6, 3), (8, 70, 69), (8, 70, 33), (2, 40, 1), (32, 3, 2)])
def test_later_tokens_have_no_part(dec, Hq, chunk, at, kv, what):
    """A token's keys and values that are NaN or infinite spoil the tokens that see it, and no other."""
    if kv == "e4m3" and what == "inf":
        pytest.skip("E4M3 has no infinity")
    L, Hkv = 150, 2
    for which in ("k", "v"):
        cache = Cache([L], Hkv, 128, kv)
        clean = Extension(cache, [chunk], Hq)
        dec.extend(clean.c)
        clean.check()
        p = L - chunk + at
        bad = 0x7f if kv == "e4m3" else float(what)
        getattr(cache, which)[int(cache.table[0, p // PAGE]), :, p % PAGE, 5:9] = bad
        x = Extension(cache, [chunk], Hq)
        dec.extend(x.c)
        torch.cuda.synchronize()
        assert torch.isfinite(x.out[:at]).all() and torch.isfinite(x.lse[:at]).all()
        assert torch.allclose(x.out[:at].float(), clean.out[:at].float(), rtol=2.0 ** -7, atol=1e-6)
        assert torch.equal(x.lse[:at], clean.lse[:at])
        if what == "nan":
            spoilt = torch.isnan(x.out[at:])
            assert (spoilt if which == "k" else spoilt[..., 5:9]).all()
        if which == "v":
            assert torch.isfinite(x.out[..., :5]).all() and torch.isfinite(x.out[..., 9:]).all()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("chunk", [5, 80])
def test_large_scores(dec, chunk, kv):
    """Scores of several hundred, of either sign: nothing overflows, and maxima that keep growing are followed."""
    cache = Cache([700], 2, 128, kv, value_scale=1.0)
    if kv == "bf16":
        ramp = torch.linspace(0.5, 12.0, PAGE * cache.table.shape[1], device=DEV).view(-1, PAGE)
        for i, page in enumerate(cache.table[0].tolist()):
            cache.k[page] *= ramp[i][None, :, None].to(torch.bfloat16)
    else:
        cache.ks *= 8.0
    run(dec, cache, [chunk], 8, "large")


@pytest.mark.parametrize("chunk", [4, 90])
def test_zero_scale_pages(dec, chunk):
    """Pages of zeros whose scale is zero too."""
    cache = Cache([140], 2, 128, "e4m3")
    for page in cache.table[0, -3:].tolist():
        cache.k[page], cache.v[page], cache.ks[page], cache.vs[page] = 0, 0, 0.0, 0.0
    run(dec, cache, [chunk], 8, "zeros")


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_offsets_beyond_32_bits(dec, kv):
    """A pool of more than 4 GB: the pages in use lie at both ends."""
    Hkv, D = 8, 128
    cache = Cache([300, 170], Hkv, D, kv)
    elements = PAGE * Hkv * D
    pages = (5 << 30) // (elements * cache.k.element_size())
    small = (cache.k, cache.v, cache.ks, cache.vs)
    where = torch.randperm(cache.pages, generator=torch.Generator().manual_seed(5))
    where = torch.where(where % 2 == 0, where, pages - 1 - where)
    big = [torch.empty((pages,) + tuple(x.shape[1:]), dtype=x.dtype, device=DEV) if x is not None else None for x in small]
    for b, x in zip(big, small):
        if x is not None:
            b[where.to(DEV)] = x
    cache.k, cache.v, cache.ks, cache.vs = big
    cache.table = torch.where(cache.table >= 0, where[cache.table.clamp(min=0).long()].to(torch.int32), cache.table)
    cache.table_dev = cache.table.to(DEV)
    cache.values = lambda which, b, n, s=small, t=cache.table: _values(s, which, t, where, b, n, Hkv, D)
    for chunks in ([3, 7], [50, 44]):
        run(dec, cache, chunks, 16, "far")
    del big
    cache.k = cache.v = None
    torch.cuda.empty_cache()


def _values(small, which, table, where, b, n, Hkv, D):
    back = {int(w): i for i, w in enumerate(where.tolist())}
    ids = torch.tensor([back[int(p)] for p in table[b, :(n + PAGE - 1) // PAGE]])
    pool, scale = (small[0], small[2]) if which == "k" else (small[1], small[3])
    x = pool.cpu()[ids]
    x = x.double() if scale is None else x.view(torch.float8_e4m3fn).double() * scale.cpu()[ids].double()[:, :, None, None]
    return x.transpose(1, 2).reshape(-1, Hkv, D)[:n]


def test_a_bound_above_the_chunks(dec):
    """The bound on the lengths may be far above them; the launch shape follows it."""
    for chunks in ([3, 5], [70, 20]):
        run(dec, Cache([90, 100], 2, 128), chunks, 8, "bound", bound=700)


def test_same_inputs_same_bytes_on_any_stream(dec):
    for chunks, lens in (([6, 3, 5], [2000, 90, 700]), ([90, 200], [1800, 400])):
        x = Extension(Cache(lens, 2, 128, "e4m3"), chunks, 8)
        dec.extend(x.c)
        x.check()
        first = (x.out.clone(), x.lse.clone())
        side = torch.cuda.Stream()
        for _ in range(3):
            x.out.fill_(float("nan"))
            side.wait_stream(torch.cuda.current_stream())
            dec.extend(x.c, stream=side)
            side.synchronize()
            assert torch.equal(first[0].view(torch.int16), x.out.view(torch.int16)) and torch.equal(first[1], x.lse)


def test_graph_replays_read_what_the_buffers_hold(dec):
    cache = Cache([900, 300, 64], 2, 128)
    x = Extension(cache, [5, 40, 9], 8)
    dec.extend(x.c)
    x.check("eager")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dec.extend(x.c, stream=stream)
    for i in range(3):
        x.q_host = normal(tuple(x.q.shape), 500 + i)
        x.q.copy_(x.q_host)
        x.totals = [900 - 100 * i, 300 - 7 * i, 64]
        x.after.copy_(torch.tensor(x.totals, dtype=torch.int32))
        x.out.fill_(float("nan"))
        graph.replay()
        x.check("replay %d" % i)


def test_workspace_is_checked(dec):
    x = Extension(Cache([6000], 2, 128), [5], 8)
    need = ra.rollout_attn_extend_workspace_size(dec.ctx, x.c)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    for at, size, status in ((ws.data_ptr(), need - 1, ra.RA_ERR_WORKSPACE_TOO_SMALL), (0, need, ra.RA_ERR_INVALID_ARG),
                             (ws.data_ptr() + 16, need, ra.RA_ERR_INVALID_ARG)):
        with pytest.raises(ra.RolloutAttnError) as e:
            ra.rollout_attn_extend(dec.ctx, x.c, ctypes.c_void_p(at), size, None)
        assert e.value.status == status
    torch.cuda.synchronize()
    assert torch.isnan(x.out.float()).all()
    ra.rollout_attn_extend(dec.ctx, x.c, ctypes.c_void_p(ws.data_ptr()), need, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    x.check()


def test_nothing_to_do(dec):
    cache = Cache([40], 2, 128)
    x = Extension(cache, [5], 8)
    for change in (dict(num_seqs=0), dict(total_tokens=0), dict(max_chunk_len=0)):
        for k, v in change.items():
            old = getattr(x.c, k)
            setattr(x.c, k, v)
            dec.extend(x.c)
            setattr(x.c, k, old)
    torch.cuda.synchronize()
    assert torch.isnan(x.out.float()).all()
