"""Plain forms of both ends of a step, sequence by sequence on the host in whole numbers and 64 bits, from the definitions in
include/rollout_attn_step.h, and batches of them on the device."""
import math

import numpy as np
import torch

import paper_2507_01663_amd as ra

PAGE = 16
DEV = "cuda:0"


def ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32).reshape(-1), dtype=torch.int32, device=DEV)


def pages_of(n):
    return -(-n // PAGE)


# ---- pages --------------------------------------------------------------------------------------------

def prefix_of(b, groups):
    """The shared pages of sequence b: a list of page ids.  groups: (group of each sequence, offsets, pages) or None."""
    if groups is None:
        return []
    g = int(groups[0][b])
    if g < 0 or g >= len(groups[1]) - 1:
        return []
    return [int(x) for x in groups[2][int(groups[1][g]):int(groups[1][g + 1])]]


def place(lens, asked, held, table, stack, free, room, groups=None):
    """What ra_place says: a dict of numpy arrays (table: a copy)."""
    table, M = np.array(table), table.shape[1]
    free = min(max(free, 0), len(stack))
    top, wanted, tokens = free, 0, 0
    lens_out, held_out, cu, positions, slots, seqs = list(lens), list(held), [0], [], [], []
    for b, (L, n, h) in enumerate(zip(map(int, lens), map(int, asked), map(int, held))):
        shared = prefix_of(b, groups)
        H, P = max(h, len(shared)), pages_of(L + n)
        if n > 0 and L >= 0 and h >= 0 and H <= M and P <= M and L <= PAGE * H:
            more = max(0, P - H)
            wanted, tokens = wanted + more, tokens + n
            if (more == 0 or wanted <= free) and tokens <= room:
                table[b, h:H] = shared[h:H]
                for i in range(H, P):
                    top -= 1
                    table[b, i] = stack[top]
                lens_out[b], held_out[b] = L + n, max(H, P)
                for p in range(L, L + n):
                    positions.append(p), slots.append(int(table[b, p // PAGE]) * PAGE + p % PAGE), seqs.append(b)
        cu.append(len(positions))
    rest = [-1] * (room - len(positions))
    i32 = lambda x: np.array(x, dtype=np.int32)
    return dict(block_table=table, cu_seqlens=i32(cu), lens_out=i32(lens_out), held_out=i32(held_out), free_count_out=i32([top]),
                positions=i32(positions + rest), slots=np.array(slots + rest, dtype=np.int64), seqs=i32(seqs + rest))


def release(keep, held, table, stack, free, groups=None):
    stack, held_out, M = np.array(stack), np.array(held, dtype=np.int32), table.shape[1]
    at = min(max(free, 0), len(stack))
    for b, (k, h) in enumerate(zip(map(int, keep), map(int, held))):
        if 0 <= h <= M:
            K = min(h, pages_of(max(k, 0)))
            held_out[b] = K
            for i in range(max(K, len(prefix_of(b, groups))), h):
                if at < len(stack):
                    stack[at] = table[b, i]
                    at += 1
    return dict(held_out=held_out, free_pages=stack, free_count_out=np.array([at], dtype=np.int32))


class Placing:
    """A call of place on the device.  alias: lengths, counts and the stack's height are written where they are read."""

    def __init__(self, lens, asked, held, table, stack, free, room, groups=None, alias=False, tokens=True):
        self.want = place(lens, asked, held, table, stack, free, room, groups)
        n = len(lens)
        self.lens, self.asked, self.held, self.stack, self.free = (ints(x) for x in (lens, asked, held, stack, [free]))
        junk = lambda k, kind=torch.int32: torch.full((k,), -77, dtype=kind, device=DEV)
        self.got = dict(block_table=torch.tensor(table, dtype=torch.int32, device=DEV), cu_seqlens=junk(n + 1), lens_out=self.lens if alias else junk(n),
                        held_out=self.held if alias else junk(n), free_count_out=self.free if alias else junk(1))
        if tokens:
            self.got.update(positions=junk(room), slots=junk(room, torch.int64), seqs=junk(room))
        self.groups = None if groups is None else [ints(x) for x in groups]
        hint = {} if groups is None else dict(zip(("seq_group", "prefix_page_offsets", "prefix_pages"), self.groups))
        g = self.got
        self.c = ra.place_from_tensors(self.lens, self.asked, self.held, g["block_table"], self.stack, self.free, g["cu_seqlens"], g["lens_out"],
                                       g["held_out"], g["free_count_out"], g.get("positions"), g.get("slots"), g.get("seqs"), room, **hint)

    def check(self, what=""):
        torch.cuda.synchronize()
        for name, x in self.got.items():
            assert np.array_equal(x.cpu().numpy(), self.want[name]), (what, name)
        return self


class Releasing:
    def __init__(self, keep, held, table, stack, free, groups=None, alias=False):
        self.want = release(keep, held, table, stack, free, groups)
        self.keep, self.held, self.free = ints(keep), ints(held), ints([free])
        self.table = torch.tensor(table, dtype=torch.int32, device=DEV)
        junk = lambda k: torch.full((k,), -77, dtype=torch.int32, device=DEV)
        self.got = dict(held_out=self.held if alias else junk(len(keep)), free_pages=ints(stack), free_count_out=self.free if alias else junk(1))
        self.groups = None if groups is None else [ints(x) for x in groups]
        hint = {} if groups is None else dict(zip(("seq_group", "prefix_page_offsets"), self.groups))
        self.c = ra.release_from_tensors(self.keep, self.held, self.table, self.got["free_pages"], self.free, self.got["held_out"],
                                         self.got["free_count_out"], **hint)

    check = Placing.check


def batch(seed, n, most=400, new=60, spare=0.2, group=0, prefix=0, slack=1.0):
    """A batch of n sequences with random lengths over randomly placed pages: (lens, asked, held, table, stack, free, groups).  slack: pages
    on the stack for each that is wanted."""
    r = np.random.default_rng(seed)
    lens, asked = r.integers(0, most + 1, n), r.integers(0, new + 1, n)
    groups, shared = None, 0
    if group:
        shared = prefix
        of = np.arange(n) // group
        of[r.random(n) < 0.15] = -1
        lens = np.where(of >= 0, np.maximum(lens, prefix * PAGE), lens)
        count = int(of.max()) + 1 if n else 0
        groups = [of, np.arange(count + 1) * prefix, None]
    held = np.array([pages_of(int(x)) for x in lens]) + (r.random(n) < spare) * r.integers(1, 3, n)
    if group:
        fresh = (groups[0] >= 0) & (lens == prefix * PAGE)
        held = np.where(fresh, r.integers(0, prefix + 1, n), held)
    mine = [max(0, int(h) - (shared if group and groups[0][b] >= 0 else 0)) for b, h in enumerate(held)]
    need = int(sum(max(0, pages_of(int(a + b)) - int(h)) for a, b, h in zip(lens, asked, held)))
    free = int(need * slack) + (2 if slack >= 1 else 0)
    extra = (len(groups[1]) - 1) * prefix if group else 0
    ids = r.permutation(sum(mine) + free + extra + 5)
    M = max([1] + [max(int(h), pages_of(int(a + b)), shared) for a, b, h in zip(lens, asked, held)])
    table = np.full((n, M), -1, dtype=np.int32)
    at = 0
    if group:
        groups[2] = ids[:extra]
        at = extra
    for b in range(n):
        own = prefix_of(b, groups)[:int(held[b])]
        table[b, :len(own)] = own
        k = int(held[b]) - len(own)
        table[b, len(own):len(own) + k] = ids[at:at + k]
        at += k
    stack = np.full(len(ids), -1, dtype=np.int32)
    stack[:free] = ids[at:at + free]
    return lens, asked, held, table, stack, free, groups


# ---- verification -------------------------------------------------------------------------------------

def distribution(x, T):
    """softmax(x / T) in 64 bits, None if the row has none.  x: float64 [V]."""
    if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
        return None
    if not T > 0:
        p = np.zeros_like(x)
        p[int(np.argmax(x))] = 1.0
        return p
    T = min(max(float(T), float(np.float32(1e-30))), float(np.float32(1e30)))
    with np.errstate(over="ignore"):
        e = np.exp((x - x.max()) / T)
    return e / e.sum()


def pick(w, v):
    """The first i with w_0 + .. + w_i > v * sum(w)."""
    v = 0.0 if np.isnan(v) else min(max(float(v), 0.0), 1.0)
    c = np.cumsum(w)
    over = np.flatnonzero(c > v * c[-1])
    return int(over[0]) if over.size else int(np.flatnonzero(w > 0)[-1])


def verify(logits, cu, tokens, u, v, T=None, draft=None, draft_rows=None):
    """What ra_verify says, rows given in 64 bits: (accepted, out_tokens, out_logprobs, next); rows of no sequence are None in both."""
    R, V = logits.shape
    out, lps, accepted, nexts = [None] * R, [None] * R, [], []
    for b in range(len(cu) - 1):
        first, end, t = int(cu[b]), int(cu[b + 1]), 1.0 if T is None else float(T[b])
        if first < 0 or end > R or first >= end:
            accepted.append(0), nexts.append(-1)
            continue
        for row in range(first, end):
            out[row], lps[row] = -1, 0.0
        for row in range(first, end):
            p, x = distribution(logits[row], t), int(tokens[row + 1]) if row + 1 < end else -1
            if p is None:
                out[row], lps[row] = -1, math.nan
                break
            w = p
            if 0 <= x < V:
                if draft is None:
                    q = np.zeros(V)
                    q[x] = 1.0
                elif not t > 0:
                    q = np.zeros(V)
                else:
                    d = int(draft_rows[b]) + row - first
                    q = distribution(draft[d], t) if 0 <= d < len(draft) else None
                if q is not None:
                    if (p[x] == 1.0) if not t > 0 else float(u[row]) * q[x] < p[x]:
                        out[row], lps[row] = x, math.log(p[x])
                        continue
                    w = np.maximum(p - q, 0.0)
                    if not w.sum() > 0:
                        w = p
            i = int(np.argmax(p)) if not t > 0 else pick(w, float(v[b]))
            out[row], lps[row] = i, math.log(p[i])
            break
        accepted.append(row - first), nexts.append(out[row])
    return accepted, out, lps, nexts


class Verifying:
    """A batch of rows on the device.  exact: all sums are binary64 (the library's choice for few logits).  rows: rows of each sequence; behind: rows of nobody at the end; logits, draft: float64 [R, V] that
    are values of their types.  pad: elements between two rows; shift: elements before the first."""

    def __init__(self, rows, logits, tokens, u, v, T=None, draft=None, draft_rows=None, dtype="bf16", draft_dtype=None, pad=0, shift=0, lead=0):
        self.rows, self.cu_host = rows, np.concatenate([[lead], lead + np.cumsum(rows)]).astype(np.int32)
        R, V = logits.shape
        single = lambda x: None if x is None else np.asarray(x, dtype=np.float32).astype(np.float64)
        u, v, T = single(u), single(v), single(T)                # (what the device gets)
        self.host = (logits, self.cu_host, tokens, u, v, T, draft, draft_rows)
        self.logits = self._device(logits, dtype, pad, shift)
        self.draft = None if draft is None else self._device(draft, draft_dtype or dtype, pad, shift)
        f = lambda x: None if x is None else torch.tensor(np.asarray(x, dtype=np.float32), device=DEV)
        self.cu, self.tokens, self.u, self.v, self.T = ints(self.cu_host), ints(tokens), f(u), f(v), f(T)
        self.draft_rows = None if draft_rows is None else ints(draft_rows)
        n = len(rows)
        self.accepted, self.next, self.out = (torch.full((k,), -77, dtype=torch.int32, device=DEV) for k in (n, n, R))
        self.lps = torch.full((R,), 77.0, device=DEV)
        self.c = ra.verify_from_tensors(self.logits, self.cu, self.tokens, self.u, self.v, self.accepted, self.out, self.lps, self.next, self.T,
                                        self.draft, self.draft_rows)

    exact = True

    @staticmethod
    def _device(x, dtype, pad, shift):
        kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        R, V = x.shape
        flat = torch.full((shift + R * (V + pad) + 64,), float("nan"), dtype=kind, device=DEV)   # what lies between rows is nobody's
        rows = flat[shift:shift + R * (V + pad)].view(R, V + pad)[:, :V]
        rows.copy_(torch.from_numpy(x).to(kind))
        return rows

    def check(self, what=""):
        """Tokens and counts are those of the reference.  A log-probability is rounded once to binary32 (2^-24 of it); beside that the
        weights' 2^-38 in the sum of a row, and binary64 steps in (l - top) / T of a size up to 1e4 (1e4 2^-52).  A row's sum of binary32
        weights w = 2^y is off by (3 ln 2 |y| + 2) 2^-24 w for each (the difference, the factor and the product are rounded, and the
        power's step) and 3 2^-24 for adding eight up; y is against a value up to 8 below the largest, and sum(w |y|) <= log2(V)
        sum(w) where the largest weighs 1 (the entropy in bits): (3 ln 2 (log2(V) + 8) + 5) 2^-24 of the sum, 5.7e-5 2^-4 = 3.6e-6 for
        V = 2^17, and as much in its logarithm."""
        sums = 0.0 if self.exact else 1.05 * (3 * math.log(2) * (math.log2(max(2, self.c.vocab)) + 8) + 5) * 2.0 ** -24
        torch.cuda.synchronize()
        accepted, out, lps, nexts = verify(*self.host)
        assert self.accepted.tolist() == accepted, (what, self.accepted.tolist(), accepted)
        assert self.next.tolist() == nexts, (what, self.next.tolist(), nexts)
        got, glp = self.out.tolist(), self.lps.double().tolist()
        for t, (x, lp) in enumerate(zip(out, lps)):
            if x is None:
                assert got[t] == -77 and glp[t] == 77.0, (what, t)
                continue
            assert got[t] == x, (what, t, got[t], x)
            if math.isnan(lp):
                assert math.isnan(glp[t]), (what, t)
            else:
                assert abs(glp[t] - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -37 + sums, (what, t, glp[t], lp)
        return self


def rounded(x, dtype):
    """x (float64) as values of the type."""
    return torch.from_numpy(x).to(torch.bfloat16 if dtype == "bf16" else torch.float32).double().numpy()


def rows_of(seed, R, V, dtype, scale=3.0):
    return rounded(np.random.default_rng(seed).normal(0.0, scale, (R, V)), dtype)


def drafting(seed, rows, V, dtype="bf16", drafts="logits", T=None, near=0.7, draft_dtype=None, **more):
    """A batch: target rows, a draft model near to it (drafts drawn from it) or guesses."""
    r = np.random.default_rng(seed)
    R, n = int(sum(rows)) + more.get("lead", 0) + more.pop("behind", 0), len(rows)
    logits = rows_of(seed + 1, R, V, dtype)
    cu = more.get("lead", 0) + np.concatenate([[0], np.cumsum(rows)])
    tokens = r.integers(0, V, R)
    draft, starts, at = None, None, 0
    if drafts == "logits":
        draft, starts = [], []
        for b in range(n):
            starts.append(at)
            for t in range(int(cu[b]), int(cu[b + 1]) - 1):
                d = rounded(logits[t] + r.normal(0.0, near, V), draft_dtype or dtype)
                q = distribution(d, 1.0 if T is None else T[b])
                tokens[t + 1] = pick(q, r.random())
                draft.append(d)
                at += 1
        draft = np.array(draft).reshape(at, V)
    else:
        for b in range(n):
            for t in range(int(cu[b]), int(cu[b + 1]) - 1):
                if r.random() < 0.6:
                    tokens[t + 1] = pick(distribution(logits[t], 1.0 if T is None else T[b]), r.random())
    f32 = lambda k: r.random(k).astype(np.float32)
    return Verifying(rows, logits, tokens, f32(R), f32(n), T, draft, starts, dtype, draft_dtype, **more)
