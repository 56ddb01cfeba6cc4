"""Norm and rotation of query and key rows, and the append of chunks of new tokens to the paged cache, on the GPU, against the
64-bit reference."""
import numpy as np
import pytest
import torch

import paper_2507_01663_amd as ra
from chunk_util import DEV, PAGE, U, Cache, cu_of, ints, normal, rotated
from workload.gen import e4m3_encode

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def dec():
    d = ra.Decoder(0)
    yield d
    d.close()


def close(got, ref, scale=None):
    """One rounding to bf16 of a binary32 result: U of the value, and binary32 errors in proportion to the row's size."""
    row = ref.abs().amax(dim=-1, keepdim=True)
    err = (got.double().cpu() - ref).abs() - 1.01 * U * ref.abs() - 4e-6 * row - 1e-30
    assert err.max() <= 0, float(err.max())


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16 if a.element_size() == 2 else torch.uint8),
                       b.contiguous().view(torch.int16 if b.element_size() == 2 else torch.uint8))


def weights(D, seed):
    g = torch.Generator().manual_seed(seed)
    return 1.0 + 0.3 * torch.randn(D, generator=g), 1.0 + 0.3 * torch.randn(D, generator=g)


def packed(T, Hq, Hkv, D, seed):
    """One projection's output: views of its query, key and value parts."""
    x = normal((T, (Hq + 2 * Hkv) * D), seed).to(DEV)
    return x, x[:, :Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), x[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))


HEADS = [(4, 2, 64), (1, 1, 64), (32, 2, 64), (28, 4, 128), (3, 1, 128), (64, 8, 128), (16, 16, 64)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("T", [1, 2, 7, 65])
@pytest.mark.parametrize("norm", [True, False])
def test_rotate(dec, T, Hq, Hkv, D, norm):
    for rot in (D, D // 2, 16, D - 16, 0):
        for inter in (False, True):
            print("case T", T, "heads", Hq, Hkv, D, "rot", rot, inter, flush=True)
            _, q, k, _ = packed(T, Hq, Hkv, D, seed=T + rot)
            pos = torch.randint(0, 50, (T,), generator=torch.Generator().manual_seed(T)).to(torch.int32)
            rope = ra.rope_table(50, rot, 1e4, "cpu") if rot else None
            qw, kw = weights(D, rot) if norm else (None, None)
            qo, ko = (torch.full((T, h, D), float("nan"), dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv))
            on = lambda x: None if x is None else x.to(DEV)
            there = [on(x) for x in (pos, rope, qw, kw)]
            dec.rotate(ra.rotate_from_tensors(q, k, qo, ko, *there, eps=EPS, interleaved=inter))
            torch.cuda.synchronize()
            close(qo, rotated(q.double().cpu(), qw, pos, rope, EPS, inter))
            close(ko, rotated(k.double().cpu(), kw, pos, rope, EPS, inter))
            if not norm and rot < D:
                assert same_bits(qo[..., rot:], q[..., rot:])


def test_rotate_many_rows_in_place_and_one_tensor(dec):
    """As many rows as make a wave take four passes; in place; queries or keys alone; a weight for one of the two."""
    T, Hq, Hkv, D = 9001, 28, 4, 128
    x, q, k, v = packed(T, Hq, Hkv, D, 3)
    pos = torch.arange(T, dtype=torch.int32)
    rope = ra.rope_table(T, D, 1e6, "cpu")
    qw, kw = weights(D, 1)
    was = x.clone()
    qo, ko = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV), torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=DEV)
    args = dict(positions=pos.to(DEV), rope=rope.to(DEV), q_weight=qw.to(DEV), k_weight=kw.to(DEV))
    dec.rotate(ra.rotate_from_tensors(q, k, qo, ko, **args))
    some = torch.cat([torch.arange(0, 40), torch.arange(T - 40, T)])
    close(qo[some], rotated(q[some].double().cpu(), qw, pos[some], rope))
    close(ko[some], rotated(k[some].double().cpu(), kw, pos[some], rope))
    dec.rotate(ra.rotate_from_tensors(q, None, q, None, **args))         # in place, the queries
    torch.cuda.synchronize()
    assert same_bits(q, qo) and same_bits(x[:, Hq * D:], was[:, Hq * D:])
    args["q_weight"] = None
    dec.rotate(ra.rotate_from_tensors(None, k, None, k, **args))
    torch.cuda.synchronize()
    assert same_bits(k, ko) and same_bits(x[:, (Hq + Hkv) * D:], was[:, (Hq + Hkv) * D:])


def test_positions_out_of_the_table_are_left_out(dec):
    T, Hq, Hkv, D = 6, 4, 2, 64
    _, q, k, _ = packed(T, Hq, Hkv, D, 9)
    pos = torch.tensor([0, -1, 9, 10, 2 ** 31 - 1, 3], dtype=torch.int32)
    rope = ra.rope_table(10, D, 1e4, "cpu")
    qo, ko = (torch.full((T, h, D), 7.0, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv))
    dec.rotate(ra.rotate_from_tensors(q, k, qo, ko, positions=pos.to(DEV), rope=rope.to(DEV)))
    torch.cuda.synchronize()
    fine = [0, 2, 5]
    close(qo[fine], rotated(q[fine].double().cpu(), None, pos[fine], rope))
    close(ko[fine], rotated(k[fine].double().cpu(), None, pos[fine], rope))
    assert (qo[[1, 3, 4]] == 7).all() and (ko[[1, 3, 4]] == 7).all()


def test_odd_rows(dec):
    """Rows of zeros, very large and very small rows, a NaN: what the formula says, and no effect on other rows."""
    T, Hq, Hkv, D = 5, 2, 1, 128
    q, k = normal((T, Hq, D), 1), normal((T, Hkv, D), 2)
    q[1], q[2], q[3] = 0.0, q[2] * 1e15, q[3] * 1e-15
    q[4, 0, 3] = float("nan")
    qw, kw = weights(D, 2)
    qo, ko = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV), torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=DEV)
    dec.rotate(ra.rotate_from_tensors(q.to(DEV), k.to(DEV), qo, ko, q_weight=qw.to(DEV), k_weight=kw.to(DEV), eps=EPS))
    torch.cuda.synchronize()
    none = torch.zeros(T, dtype=torch.int32)
    close(qo[:4], rotated(q[:4].double(), qw, none, None, EPS))
    assert (qo[1] == 0).all() and torch.isnan(qo[4, 0]).all()
    close(qo[4:, 1:], rotated(q[4:, 1:].double(), qw, none, None, EPS))


# ---- append -------------------------------------------------------------------------------------------------


class Append:
    def __init__(self, chunks, before, heads, kv="bf16", rot=None, norm=True, inter=False, positions=None, layout="hpd", with_q=True, seed=0,
                 value_scale=1.0, rope_len=4000):
        Hq, Hkv, D = heads
        self.chunks, self.before, self.inter = list(chunks), list(before), inter
        T = sum(chunks)
        self.cache = Cache(before, Hkv, D, kv, seed=seed, layout=layout, room=max(chunks))
        self.x, self.q, self.k, self.v = packed(T, Hq, Hkv, D, 50 + seed)
        if value_scale != 1.0:
            self.x.mul_(value_scale)
        rot = D if rot is None else rot
        self.rope = ra.rope_table(rope_len, rot, 1e4, "cpu") if rot else None
        self.qw, self.kw = weights(D, seed) if norm else (None, None)
        self.where = torch.cat([torch.arange(b, b + n) for b, n in zip(before, chunks)] or [torch.zeros(0)]).to(torch.int32)
        self.positions = self.where if positions is None else positions
        self.q_out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV) if with_q else None
        on = lambda t: None if t is None else t.to(DEV)
        c = self.cache
        self.pools = [None if t is None else t.clone() for t in (c.k, c.v, c.ks, c.vs)]      # as they were
        # (a descriptor has addresses; the tensors have to stay)
        self.cu, self.lens, self.turn = cu_of(chunks), ints(before), [on(t) for t in (positions, self.rope, self.qw, self.kw)]
        self.c = ra.append_chunk_from_tensors(self.k, self.v, self.cu, max(chunks), c.table_dev, self.lens, c.k, c.v, k_scale=c.ks, v_scale=c.vs,
                                              q=self.q if with_q else None, q_out=self.q_out, positions=self.turn[0], rope=self.turn[1],
                                              q_weight=self.turn[2], k_weight=self.turn[3], eps=EPS, interleaved=inter)

    def check(self):
        torch.cuda.synchronize()
        c = self.cache
        if self.q_out is not None:
            close(self.q_out, rotated(self.q.double().cpu(), self.qw, self.positions, self.rope, EPS, self.inter))
        k = rotated(self.k.double().cpu(), self.kw, self.positions, self.rope, EPS, self.inter)
        v = self.v.double().cpu()
        for pool, was, scale, old_scale, rows, turned in ((c.k, self.pools[0], c.ks, self.pools[2], k, True), (c.v, self.pools[1], c.vs, self.pools[3], v, False)):
            pool, was = pool.cpu(), was.cpu()
            expected_same = torch.ones(pool.shape[0], PAGE, dtype=torch.bool)
            t = 0
            for b, n in enumerate(self.chunks):
                at, end = self.before[b], self.before[b] + n
                while at < end:
                    page, slot = int(c.table[b, at // PAGE]), at % PAGE
                    take = min(PAGE - slot, end - at)
                    new = rows[t:t + take].transpose(0, 1)                # [Hkv, take, D]
                    got = pool[page, :, slot:slot + take]
                    expected_same[page, slot:slot + take] = False
                    if scale is None:
                        if turned:
                            close(got, new)
                        else:
                            assert torch.equal(got.double(), new)
                    else:
                        self.check_page(page, slot, take, new, pool, was, scale.cpu(), old_scale.cpu(), expected_same)
                    at, t = at + take, t + take
            bits = torch.int16 if scale is None else torch.uint8
            same = (pool.view(bits) == was.view(bits)).all(dim=(1, 3))
            assert same[expected_same].all()
        return self

    @staticmethod
    def check_page(page, slot, take, new, pool, was, scale, old_scale, expected_same):
        """Scale and codes: half a unit of E4M3 of what they stand for, in units of the scale; a hundredth more for binary32."""
        top = new.abs().amax(dim=(1, 2))
        fresh = torch.where(top > 0, top / 448.0, torch.ones_like(top))
        old = old_scale[page].double()
        want = fresh if slot == 0 else torch.where(top <= old * 448.0, old, fresh)
        assert torch.allclose(scale[page].double(), want, rtol=1e-6, atol=0)
        s = scale[page].double()[:, None, None]

        def near(codes, x):
            y = (x / s).abs()
            err = (codes.view(torch.float8_e4m3fn).double() * s - x).abs() / s - 1.01 * torch.maximum(y * 2.0 ** -4, torch.full_like(y, 2.0 ** -10))
            assert err.max() <= 0, float(err.max())

        near(pool[page, :, slot:slot + take].contiguous(), new)
        if slot:
            kept = scale[page] == old_scale[page]
            for h in range(pool.shape[1]):
                if kept[h]:
                    assert torch.equal(pool[page, h, :slot], was[page, h, :slot])
                else:
                    x = was[page, h, :slot].contiguous().view(torch.float8_e4m3fn).double() * old[h]
                    y = (x / s[h]).abs()
                    err = (pool[page, h, :slot].contiguous().view(torch.float8_e4m3fn).double() * s[h] - x).abs() / s[h] - 1.01 * torch.maximum(y * 2.0 ** -4, torch.full_like(y, 2.0 ** -10))
                    assert err.max() <= 0
            expected_same[page, :slot] = False


CHUNKS = [([1], [0]), ([1], [17]), ([5, 0, 16, 1, 33], [3, 9, 0, 15, 31]), ([0, 0, 40, 2], [0, 5, 8, 14]), ([1] * 7, [0, 1, 15, 16, 17, 31, 40])]


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (5, 1, 64), (8, 8, 128)])
@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_append_chunk(dec, case, heads, kv):
    chunks, before = CHUNKS[case]
    for rot, norm, inter in ((None, True, False), (32, False, True), (0, True, False), (16, True, True)):
        print("case", case, heads, kv, rot, norm, inter, flush=True)
        x = Append(chunks, before, heads, kv, rot=rot, norm=norm, inter=inter, with_q=rot != 16)
        dec.append_chunk(x.c)
        x.check()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_append_chunk_scales_layouts_positions(dec, kv):
    """Rows large and small against the page's scale; strided pools; positions of the caller's."""
    chunks, before = [9, 20, 1, 3], [5, 12, 30, 15]
    for value_scale in (4.0, 0.1, 2.0 ** -70, 1e20):
        x = Append(chunks, before, (8, 2, 128), kv, norm=False, rot=0, value_scale=value_scale, with_q=False)
        dec.append_chunk(x.c)
        x.check()
    for layout in ("phd", "gaps"):
        for D in (64, 128):
            x = Append(chunks, before, (8, 2, D), kv, layout=layout, seed=3)
            dec.append_chunk(x.c)
            x.check()
    x = Append(chunks, before, (8, 2, 128), kv, positions=torch.arange(sum(chunks), dtype=torch.int32).flip(0))
    dec.append_chunk(x.c)
    x.check()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_append_many_rows(dec, kv):
    """As many tokens as make a wave take four passes, and more sequences than a wave looks at together."""
    chunks, before = [(b * 7) % 61 for b in range(300)], [(b * 13) % 50 for b in range(300)]
    x = Append(chunks, before, (2, 1, 64), kv)
    dec.append_chunk(x.c)
    x.check()
    x = Append([700, 33, 500], [40, 3, 0], (40, 8, 128), kv)
    dec.append_chunk(x.c)
    x.check()


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_one_token_gives_what_append_gives(dec, kv):
    for value_scale in (1.0, 5.0):
        before = [0, 1, 15, 16, 31, 100]
        x = Append([1] * 6, before, (8, 2, 128), kv, rot=0, norm=False, value_scale=value_scale)
        c = x.cache
        twin = [None if t is None else t.clone() for t in x.pools]
        dec.append_chunk(x.c)
        q = torch.zeros((6, 8, 128), dtype=torch.bfloat16, device=DEV)
        out, lse, lens = torch.empty_like(q), torch.empty((6, 8), device=DEV), ints(before)
        p = ra.problem_from_tensors(q, twin[0], twin[1], c.table_dev, lens, out, lse, 0.1, k_scale=twin[2], v_scale=twin[3])
        k, v = x.k.contiguous(), x.v.contiguous()
        dec.append(p, k, v)
        torch.cuda.synchronize()
        for a, b in zip((c.k, c.v, c.ks, c.vs), twin):
            assert a is None or torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_codes_are_the_nearest(dec):
    """Without norm and rotation every code is decided as the format says: those of the host's quantiser."""
    for value_scale in (1.0, 1e-4, 2.0 ** -75, 3e30):
        x = Append([16, 48], [0, 32], (4, 2, 128), "e4m3", rot=0, norm=False, with_q=False, value_scale=value_scale)
        dec.append_chunk(x.c)
        torch.cuda.synchronize()
        for pool, scale, rows in ((x.cache.k, x.cache.ks, x.k), (x.cache.v, x.cache.vs, x.v)):
            pool, scale, rows, t = pool.cpu().numpy(), scale.cpu().numpy(), rows.float().cpu().numpy(), 0
            for b, n in enumerate(x.chunks):
                for p in range(x.before[b] // PAGE, (x.before[b] + n) // PAGE):
                    page = int(x.cache.table[b, p])
                    new = rows[t:t + PAGE].transpose(1, 0, 2)
                    s = (np.abs(new).max(axis=(1, 2)) / np.float32(448.0)).astype(np.float32)
                    assert np.array_equal(scale[page], s)
                    assert np.array_equal(pool[page], e4m3_encode(new / s[:, None, None]))
                    t += PAGE


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_tokens_without_a_place_are_left_out(dec, kv):
    """Lengths and pages out of range, positions past the rotation's table: nothing is written for them, the rest is."""
    x = Append([4, 4, 4, 20], [3, 8, 5, 60], (4, 2, 64), kv, rope_len=70)
    c = x.cache
    room = c.table.shape[1] * PAGE
    lens = ints([room - 2, -3, 5, 60])
    bad = c.table.clone()
    bad[2, 0] = c.pages
    x.c.seq_lens, x.c.block_table = lens.data_ptr(), (keep := bad.to(DEV)).data_ptr()
    pages_before = [t.clone() for t in (c.k, c.v)]
    dec.append_chunk(x.c)
    torch.cuda.synchronize()
    assert keep is not None
    where = torch.cat([torch.arange(a, a + n) for a, n in ((room - 2, 4), (-3, 4), (5, 4), (60, 20))]).to(torch.int32)
    fine = ((where >= 0) & (where < 70)).nonzero().flatten()
    close(x.q_out[fine], rotated(x.q[fine].double().cpu(), x.qw, where[fine], x.rope, EPS))
    rest = [t for t in range(len(where)) if t not in fine.tolist()]
    assert torch.isnan(x.q_out[rest]).all()
    k = rotated(x.k.double().cpu(), x.kw, where.clamp(0, 69), x.rope, EPS)
    written = torch.zeros(c.pages, PAGE, dtype=torch.bool)
    for t, w in enumerate(where.tolist()):
        b = 0 if t < 4 else 1 if t < 8 else 2 if t < 12 else 3
        if b in (1, 2) or not 0 <= w < min(70, room):
            continue
        page = int(bad[b, w // PAGE])
        written[page, w % PAGE] = True
        if kv == "bf16":
            close(c.k[page, :, w % PAGE], k[t])
            assert torch.equal(c.v[page, :, w % PAGE].double().cpu(), x.v[t].double().cpu())
        else:
            s = c.ks[page].double().cpu()[:, None]
            y = (k[t] / s).abs()
            err = (c.k[page, :, w % PAGE].view(torch.float8_e4m3fn).double().cpu() * s - k[t]).abs() / s - 1.01 * torch.maximum(y * 2.0 ** -4, torch.full_like(y, 2.0 ** -10))
            assert err.max() <= 0
    untouched = ~written.any(dim=1)
    for a, b in zip((c.k, c.v), pages_before):
        assert torch.equal(a.cpu()[untouched].view(torch.uint8), b.cpu()[untouched].view(torch.uint8))


def test_append_in_place_queries_stream_and_graph(dec):
    for kv in ("bf16", "e4m3"):
        x = Append([5, 30, 1], [10, 3, 47], (8, 2, 128), kv)
        raw = x.q.clone()
        x.c.rot.q_out, x.c.rot.q_out_stride_token = x.c.rot.q, x.c.rot.q_stride_token
        dec.append_chunk(x.c)
        torch.cuda.synchronize()
        ref = rotated(raw.double().cpu(), x.qw, x.positions, x.rope, EPS)
        close(x.q, ref)
        x.c.rot.q_out, x.c.rot.q_out_stride_token = x.q_out.data_ptr(), x.q_out.stride(0)
        x.q.copy_(raw)
        first = [None if t is None else t.clone() for t in (x.cache.k, x.cache.v, x.cache.ks, x.cache.vs)]
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            dec.append_chunk(x.c, stream=stream)
        for _ in range(3):
            for t, was in zip((x.cache.k, x.cache.v, x.cache.ks, x.cache.vs), x.pools):
                if t is not None:
                    t.copy_(was)
            x.q_out.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            close(x.q_out, ref)
            for t, one in zip((x.cache.k, x.cache.v, x.cache.ks, x.cache.vs), first):
                assert t is None or torch.equal(t.contiguous().view(torch.uint8), one.contiguous().view(torch.uint8))
