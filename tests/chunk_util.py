"""Plain 64-bit forms of the operators for chunks of new tokens, and batches of them on the device.  The references work on
the host, token by token and page by page, from the definitions in include/rollout_attn_chunk.h."""
import numpy as np
import torch

import paper_2507_01663_amd as ra

PAGE = 16
DEV = "cuda:0"
U = 2.0 ** -8          # bf16 has eight significant bits: half a unit in the last place, relative


def rotated(x, weight, positions, rope, eps=1e-6, interleaved=False):
    """x [T, H, D] (64 bits) normalised (weight None: not) and rotated (rope None: not)."""
    y = x.clone()
    D = x.shape[-1]
    if weight is not None:
        y = x * weight.double() / torch.sqrt((x * x).sum(-1, keepdim=True) / D + eps)
    if rope is None or rope.shape[1] == 0:
        return y
    z, rot = y.clone(), rope.shape[1]
    for t in range(x.shape[0]):
        row = rope[int(positions[t])].double()
        for j in range(rot // 2):
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
            c, s = row[j], row[rot // 2 + j]
            z[t, :, a] = y[t, :, a] * c - y[t, :, b] * s
            z[t, :, b] = y[t, :, b] * c + y[t, :, a] * s
    return z


def attention(q, k, v, before, scale):
    """q [n, Hq, D] over k, v [S, Hkv, D] (64 bits): token i sees keys 0 .. before + i.  (out, lse, sum of weights times |v|)"""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, lse, mag = torch.zeros_like(q), torch.full((n, Hq), float("-inf"), dtype=torch.float64), torch.zeros_like(q)
    for i in range(n):
        m = min(before + i + 1, k.shape[0])
        if m <= 0:
            continue
        for h in range(Hq):
            s = (k[:m, h // G] @ q[i, h]) * scale
            top = s.max()
            w = torch.exp(s - top)
            z = w.sum()
            out[i, h] = (w[:, None] * v[:m, h // G]).sum(0) / z
            mag[i, h] = (w[:, None] * v[:m, h // G].abs()).sum(0) / z
            lse[i, h] = top + torch.log(z)
    return out, lse, mag


class Cache:
    """A paged cache on the device: sequences of the given lengths over randomly placed pages, poisoned (NaN) wherever nothing
    is stored.  layout "hpd": [page, head, slot, d]; "phd": [page, slot, head, d], given as a view; "gaps": rows with space
    between them."""

    def __init__(self, lens, Hkv, D, kv="bf16", seed=0, layout="hpd", room=0, spare=3, value_scale=1.0):
        self.g = torch.Generator().manual_seed(1000 + seed)
        self.Hkv, self.D, self.kv, self.lens = Hkv, D, kv, list(lens)
        need = [(L + room + PAGE - 1) // PAGE for L in self.lens]
        self.pages = sum(need) + spare
        ids = torch.randperm(self.pages, generator=self.g)[:sum(need)].to(torch.int32)
        self.table = torch.full((len(need), max(1, max(need, default=1))), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.k, self.ks = self._pool(value_scale, layout)
        self.v, self.vs = self._pool(value_scale, layout)
        self.table_dev = self.table.to(DEV)

    def _pool(self, value_scale, layout):
        P, H, D = self.pages, self.Hkv, self.D
        stored = torch.zeros((P, PAGE), dtype=torch.bool)
        for b, L in enumerate(self.lens):
            for t in range(L):
                stored[int(self.table[b, t // PAGE]), t % PAGE] = True
        x = (value_scale * torch.randn((P, H, PAGE, D), generator=self.g)).to(torch.bfloat16)
        scale = None
        if self.kv == "bf16":
            x[~stored[:, None].expand(P, H, PAGE)] = float("nan")
            data = x
        else:
            scale = x.float().abs().amax(dim=(2, 3)) / 448.0 * (0.5 + torch.rand((P, H), generator=self.g))
            data = (x.float() / scale[:, :, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
            data[~stored[:, None].expand(P, H, PAGE)] = 0x7f
            scale = scale.to(DEV)
        kind = data.dtype
        if layout == "phd":
            pool = torch.empty((P, PAGE, H, D), dtype=kind, device=DEV).transpose(1, 2)
        elif layout == "gaps":
            pool = torch.empty((P, H + 1, PAGE + 1, D + 32), dtype=kind, device=DEV)[:, :H, :PAGE, :D]
        else:
            pool = torch.empty((P, H, PAGE, D), dtype=kind, device=DEV)
        pool.copy_(data)
        return pool, scale

    def values(self, which, b, n):
        """The first n stored tokens of sequence b, [n, Hkv, D] in 64 bits on the host."""
        pool, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        ids = self.table[b, :(n + PAGE - 1) // PAGE].long()
        x = pool.cpu()[ids]
        x = x.double() if scale is None else x.view(torch.float8_e4m3fn).double() * scale.cpu()[ids].double()[:, :, None, None]
        return x.transpose(1, 2).reshape(-1, self.Hkv, self.D)[:n]


def cu_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32), device=DEV)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


def normal(shape, seed, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16)


class Extension:
    """A batch of chunks over a cache: chunks[b] new tokens, the last of totals[b] (the cache's lengths unless given)."""

    def __init__(self, cache, chunks, Hq, seed=0, totals=None, q_gap=0, bound=None):
        self.cache, self.chunks, self.Hq = cache, list(chunks), Hq
        self.totals = list(cache.lens if totals is None else totals)
        T, D = sum(chunks), cache.D
        self.q_host = normal((T, Hq, D), 77 + seed)
        wide = torch.empty((T, Hq * D + q_gap), dtype=torch.bfloat16, device=DEV)
        self.q = wide[:, :Hq * D].unflatten(1, (Hq, D))
        self.q.copy_(self.q_host)
        self.out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.lse = torch.full((T, Hq), float("nan"), dtype=torch.float32, device=DEV)
        self.cu, self.after = cu_of(chunks), ints(self.totals)
        self.scale = float(np.float32(1.0 / np.sqrt(D)))
        self.c = ra.extend_from_tensors(self.q, cache.k, cache.v, self.cu, max(chunks) if bound is None else bound, cache.table_dev, self.after,
                                        self.out, self.lse, self.scale, k_scale=cache.ks, v_scale=cache.vs)

    def check(self, what=""):
        """Against the reference.  A weight and a result are each rounded once to bf16 (relative U), sums and scores are binary32:
        per element U (|out| + sum of weights |v|), a tenth more for the rest; log-sum-exp as binary32 sums of a few
        thousand products of size one."""
        torch.cuda.synchronize()
        out, lse, t = self.out.double().cpu(), self.lse.double().cpu(), 0
        for b, n in enumerate(self.chunks):
            if not n:
                continue
            L = self.totals[b]
            ref, rlse, mag = attention(self.q_host[t:t + n].double(), self.cache.values("k", b, L), self.cache.values("v", b, L), L - n, self.scale)
            got, glse = out[t:t + n], lse[t:t + n]
            assert torch.isfinite(got).all(), (what, b)
            assert torch.equal(torch.isneginf(rlse), torch.isneginf(glse)), (what, b)
            err = (got - ref).abs() - 1.1 * U * (ref.abs() + mag) - 1e-6
            assert err.max() <= 0, (what, b, float((got - ref).abs().max()), float(err.max()))
            fine = torch.isfinite(rlse)
            assert not fine.any() or (rlse - glse)[fine].abs().max() <= 1e-4, (what, b, float((rlse - glse)[fine].abs().max()))
            t += n
        return self
