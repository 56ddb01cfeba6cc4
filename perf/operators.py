"""Measured cases of the operators that serve chunks of new tokens over a paged cache, and their plain forms.

A rollout of several turns (tool output or a user's turn goes into every response), a long prompt that is taken in pieces
between decode steps, a draft of a few tokens that is checked at once: each layer of such a step normalises and rotates the
chunk's queries and keys by head, appends keys and values to the paged cache, and attends from every new token to the cache.

  rotate   norm of the rows of q and k by head (RMS, a weight per element) and rotation by position, in one pass
  append   a chunk of new tokens per sequence into the pages of the cache, keys normalised and rotated on the way, with the
           chunk's queries beside them; bf16 pools, or e4m3 pools with a scale per (page, kv head)
  extend   causal attention of every sequence's chunk over its pages, the chunk's own among them

Head shapes and lengths are those of this repository's workloads (workload/gen.py) and generic ones between and beside them.
Lengths belong to the case (they come from its "length_seed"); values, page placement and weights come from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda:0"
SLACK = 1.25                 # pages of a pool per page in use, as a serving cache has spare pages
THETA = 1e6                  # base of the rotation's frequencies
EPS = 1e-6

_decoder = None


def decoder():
    """The process's one decoder (a context and its workspace), as a worker keeps it."""
    global _decoder
    if _decoder is None:
        import paper_2507_01663_amd as ra
        _decoder = ra.Decoder(0)
    return _decoder


# ---- the cases ----------------------------------------------------------------------------------------

def _case(name, kind, heads, seqs, chunk, context, kv="bf16", singles=0, rot=None, norm=True, interleaved=False, length_seed=0):
    """chunk, context: (least, most) new tokens and tokens already cached; singles: sequences that have one new token."""
    Hq, Hkv, D = heads
    return {"name": name, "kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "seqs": seqs, "chunk_lo": chunk[0], "chunk_hi": chunk[1],
            "context_lo": context[0], "context_hi": context[1], "kv": kv, "singles": singles, "rot": D if rot is None else rot,
            "norm": norm, "interleaved": interleaved, "length_seed": length_seed}


def listed():
    return [
        # the next token of a handful of sequences, a call that is all latency
        _case("rotate_one_token", "rotate", (28, 4, 128), 4, (1, 1), (30, 700)),
        # the prompts of the 7B-shaped GRPO batch, straight from the projection's output
        _case("rotate_prompts", "rotate", (28, 4, 128), 32, (512, 512), (0, 0)),
        # a small model that rotates half of a head, in pairs of neighbours, and has no norm; ragged chunks
        _case("rotate_partial_d64", "rotate", (32, 2, 64), 23, (1, 611), (0, 2000), rot=32, norm=False, interleaved=True),
        # the cache write of a decode step of the 7B-shaped batch: one token per sequence, queries beside it
        _case("append_step", "append", (28, 4, 128), 256, (1, 1), (512, 4096)),
        # a turn's tokens into a quantised cache: chunks that start and end inside pages
        _case("append_turns_e4m3", "append", (40, 8, 128), 64, (1, 190), (1, 900), kv="e4m3"),
        # pieces of long prompts of the 72B-shaped batch into the cache
        _case("append_prompts", "append", (64, 8, 128), 16, (512, 512), (0, 1024)),
        # one short turn of a small model: a smoke run, an interactive session
        _case("extend_one_turn", "extend", (4, 2, 64), 1, (17, 17), (500, 500)),
        # drafts of five tokens checked at once, in the middle of the 7B-shaped batch
        _case("extend_drafts", "extend", (28, 4, 128), 64, (5, 5), (512, 4000)),
        # a turn's tokens for every response of a batch, ragged
        _case("extend_turns", "extend", (40, 8, 128), 40, (20, 300), (1024, 4000)),
        # the last piece of one long prompt of the 72B-shaped batch
        _case("extend_long_prompt", "extend", (64, 8, 128), 1, (2048, 2048), (14000, 14000)),
        # decode steps with two pieces of prompts among them, quantised cache
        _case("extend_mixed_e4m3", "extend", (28, 4, 128), 50, (290, 410), (256, 2600), kv="e4m3", singles=48),
        # a small model's batch: short turns, some sequences without one, some without a context, quantised cache
        _case("extend_short_turns_d64_e4m3", "extend", (32, 2, 64), 96, (0, 40), (0, 2000), kv="e4m3"),
    ]


HEADS = [(4, 2, 64), (8, 2, 64), (32, 2, 64), (28, 4, 128), (40, 8, 128), (64, 8, 128), (8, 8, 128)]


def _spread(rng, lo, hi):
    """An integer of lo .. hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "append", "extend", "extend", "extend", "extend"])
    while True:
        heads = rng.choice(HEADS)
        D = heads[2]
        most = _spread(rng, 1, 2048)
        least = rng.choice([0, 1, most, rng.randint(0, most)])
        deep = _spread(rng, 1, 15000)
        seqs = _spread(rng, 1, 300)
        c = _case("", kind, heads, seqs, (min(least, most), most), (rng.choice([0, deep // 2, deep]), deep),
                  kv=rng.choice(["bf16", "e4m3"]) if kind != "rotate" else "bf16", singles=rng.choice([0, 0, 0, seqs // 2, seqs]),
                  rot=rng.choice([D, D, D, D // 2, D // 4]), norm=rng.random() < 0.6, interleaved=rng.random() < 0.25,
                  length_seed=rng.randrange(1 << 30))
        n, ctx = _lengths(c)
        if kind == "extend":
            # (the plain form holds all of a batch's scores at once)
            scores = c["seqs"] * c["Hq"] * max(n) * (max(x + y for x, y in zip(n, ctx)) + PAGE)
            ok = work(c)["flops"] <= 1.0e12 and scores <= 2.2e9
        else:
            ok = sum(n) <= 16384
        # pools of half a gigabyte at most, all of which comes back from an append
        ok = ok and sum(n) > 0 and sum(_pages(x + y) for x, y in zip(n, ctx)) * c["Hkv"] * PAGE * D <= (1 << 27 if kind == "extend" else 1 << 26)
        if ok:
            del c["name"]
            return c


# ---- lengths ------------------------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, tokens cached before them) of every sequence; the sequences with one new token are spread among the others."""
    r, n = random.Random(case["length_seed"]), case["seqs"]
    new = [r.randint(case["chunk_lo"], case["chunk_hi"]) for _ in range(n)]
    for b in r.sample(range(n), case["singles"]):
        new[b] = 1
    return new, [r.randint(case["context_lo"], case["context_hi"]) for _ in range(n)]


def _pages(n):
    return (n + PAGE - 1) // PAGE


# ---- what the path cannot do without ------------------------------------------------------------------

def work(case):
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    n, ctx = _lengths(case)
    T = sum(n)
    e = 1 if case["kv"] == "e4m3" else 2
    if case["kind"] == "rotate":
        positions = len(set(p for x, c in zip(n, ctx) for p in range(c, c + x)))
        return {"bytes": 4 * T * (Hq + Hkv) * D + 4 * T + 4 * positions * case["rot"], "flops": 6 * T * (Hq + Hkv) * D}
    if case["kind"] == "append":
        touched = sum(_pages(c % PAGE + x) for x, c in zip(n, ctx))
        size = 4 * T * Hq * D + 2 * T * Hkv * D * (2 + e) + 4 * T * case["rot"] + 4 * touched
        return {"bytes": size + (8 * touched * Hkv if e == 1 else 0), "flops": 6 * T * (Hq + Hkv) * D}
    kv = sum(x + c for x, c in zip(n, ctx) if x)
    size = 2 * kv * Hkv * D * e + 4 * T * Hq * D + 4 * T * Hq + 4 * sum(_pages(x + c) for x, c in zip(n, ctx) if x)
    if e == 1:
        size += 8 * Hkv * sum(_pages(x + c) for x, c in zip(n, ctx) if x)
    return {"bytes": size, "flops": 4 * D * Hq * sum(x * c + x * (x + 1) // 2 for x, c in zip(n, ctx))}


# ---- inputs -------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(shape, g):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _pool(pages, Hkv, D, kv, g):
    """A pool of normal values: bf16, or E4M3 codes with one scale per (page, kv head)."""
    if kv == "bf16":
        return _normal((pages, Hkv, PAGE, D), g), None
    codes = torch.empty((pages, Hkv, PAGE, D), dtype=torch.uint8, device=DEV)
    scale = torch.empty((pages, Hkv), dtype=torch.float32, device=DEV)
    for a in range(0, pages, 1 << 14):
        x = _normal((min(pages - a, 1 << 14), Hkv, PAGE, D), g).float()
        s = x.abs().amax(dim=(2, 3)) / 448.0
        codes[a:a + x.shape[0]] = (x / s[:, :, None, None]).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        scale[a:a + x.shape[0]] = s
    return codes, scale


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _scale(D):
    return float(np.float32(1.0 / math.sqrt(D)))


def _rope(length, rot):
    """fp32 [length, rot]: the cosines of the rot / 2 angles of a position, then their sines."""
    angle = torch.arange(length, dtype=torch.float64, device=DEV)[:, None] * THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def prepare(case, seed):
    g = _generator(seed)
    Hq, Hkv, D, kind = case["Hq"], case["Hkv"], case["D"], case["kind"]
    new, ctx = (np.array(x, dtype=np.int64) for x in _lengths(case))
    T, B, total = int(new.sum()), case["seqs"], new + ctx
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    st = {"kind": kind, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T, "rot": case["rot"], "interleaved": case["interleaved"],
          "longest": int(new.max()), "cu": _dev(cu)}
    if kind != "extend":
        # one projection's output: a token's query heads, its key heads, its value heads
        x = _normal((T, (Hq + 2 * Hkv) * D), g)
        st["q"], st["k"] = x[:, :Hq * D].view(T, Hq, D), x[:, Hq * D:(Hq + Hkv) * D].view(T, Hkv, D)
        st["v"] = x[:, (Hq + Hkv) * D:].view(T, Hkv, D)
        st["rope"] = _rope(int(total.max()) + 1, case["rot"])
        st["qw"] = st["kw"] = None
        if case["norm"]:
            st["qw"], st["kw"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV) for _ in range(2))
        st["q_out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV)
    if kind == "rotate":
        st["k_out"] = torch.empty((T, Hkv, D), dtype=torch.bfloat16, device=DEV)
        st["positions"] = _dev((np.arange(T) - np.repeat(cu[:-1].astype(np.int64), new) + np.repeat(ctx, new)).astype(np.int32))
    else:
        pages = (total + PAGE - 1) // PAGE
        in_pool = max(int(pages.sum()) + 1, int(math.ceil(SLACK * int(pages.sum()))))
        phys = torch.randperm(in_pool, generator=g, device=DEV)[:int(pages.sum())].to(torch.int32).cpu().numpy()
        table = np.full((B, max(1, int(pages.max()))), -1, dtype=np.int32)
        table[np.arange(table.shape[1])[None, :] < pages[:, None]] = phys
        st["table"], st["before"], st["after"] = _dev(table), _dev(ctx.astype(np.int32)), _dev(total.astype(np.int32))
        st["kp"], st["ks"] = _pool(in_pool, Hkv, D, case["kv"], g)
        st["vp"], st["vs"] = _pool(in_pool, Hkv, D, case["kv"], g)
    if kind == "extend":
        st["q"] = _normal((T, Hq, D), g)
        st["out"] = torch.empty((T, Hq, D), dtype=torch.bfloat16, device=DEV)
        st["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV)
    if own:         # the call's descriptor: addresses and sizes, which a worker fills in once for its buffers
        import paper_2507_01663_amd as ra
        st["decoder"] = decoder()
        if kind == "rotate":
            st["call"] = ra.rotate_from_tensors(st["q"], st["k"], st["q_out"], st["k_out"], positions=st["positions"], rope=st["rope"],
                                                q_weight=st["qw"], k_weight=st["kw"], eps=EPS, interleaved=st["interleaved"])
        elif kind == "append":
            st["call"] = ra.append_chunk_from_tensors(st["k"], st["v"], st["cu"], st["longest"], st["table"], st["before"], st["kp"], st["vp"],
                                                      k_scale=st["ks"], v_scale=st["vs"], q=st["q"], q_out=st["q_out"], rope=st["rope"],
                                                      q_weight=st["qw"], k_weight=st["kw"], eps=EPS, interleaved=st["interleaved"])
        else:
            st["call"] = ra.extend_from_tensors(st["q"], st["kp"], st["vp"], st["cu"], st["longest"], st["table"], st["after"], st["out"],
                                                st["lse"], _scale(D), k_scale=st["ks"], v_scale=st["vs"])
    return st


# ---- the plain forms ----------------------------------------------------------------------------------

def _turned(x, w, positions, rope, rot, interleaved):
    """x [T, H, D] in 32 bits, normalised with weight w (None: as it is) and rotated by its token's position."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w
    cos, sin = rope[positions.long()].view(-1, 1, 2, rot // 2).unbind(2)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    y = (a * cos - b * sin, b * cos + a * sin)
    return torch.cat([torch.stack(y, dim=-1).flatten(-2) if interleaved else torch.cat(y, dim=-1), x[..., rot:]], dim=-1)


def _tokens(cu, T):
    """(sequence, place in its chunk) of each of the T tokens."""
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), t.to(torch.int32), right=True)
    return b, t - cu[b]


def _plain_write(pool, scale, rows, table, before, cu, longest):
    """rows [T, Hkv, D] in 32 bits into their pages.  In a quantised pool a page that the chunk begins gets the scale of its
    largest new value; one that it goes on with keeps its scale if the new values fit, or its old rows are brought to theirs."""
    T, Hkv, D = rows.shape
    b, i = _tokens(cu, T)
    at = before[b].long() + i
    if scale is None:
        pool[table[b, at // PAGE].long(), :, at % PAGE] = rows.to(pool.dtype)
        return
    B, P = before.numel(), (longest + PAGE - 2) // PAGE + 1         # pages that a chunk touches, at most
    first = before.long() // PAGE
    end = before.long() + (cu[1:] - cu[:-1]).long()
    logical = first[:, None] + torch.arange(P, device=DEV)
    touched = logical * PAGE < end[:, None]
    touched &= (end > before)[:, None]
    new = torch.zeros((B, P, PAGE, Hkv, D), device=DEV)
    new[b, at // PAGE - first[b], at % PAGE] = rows
    new = new.transpose(2, 3)[touched]                              # [pages, Hkv, PAGE, D]
    page = table.gather(1, logical.clamp(max=table.shape[1] - 1)).long()[touched]
    token = (logical[:, :, None] * PAGE + torch.arange(PAGE, device=DEV))[touched]
    start = before.long()[:, None].expand(B, P)[touched]
    is_old, is_new = token < start[:, None], (token >= start[:, None]) & (token < end[:, None].expand(B, P)[touched][:, None])
    old_scale, codes = scale[page], pool[page].view(torch.float8_e4m3fn).float()
    top = (new.abs() * is_new[:, None, :, None]).amax(dim=(2, 3))
    fresh = torch.where(top > 0, top / 448.0, torch.ones_like(top))
    keeps = is_old.any(dim=1)[:, None] & (top <= old_scale * 448.0)
    s = torch.where(keeps, old_scale, fresh)
    was = torch.where(keeps[:, :, None, None], codes, codes * old_scale[:, :, None, None] / s[:, :, None, None])
    y = torch.where(is_new[:, None, :, None], new / s[:, :, None, None], torch.where(is_old[:, None, :, None], was, codes))
    pool[page] = y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    scale[page] = s


def _plain_extend(st):
    T, Hq, Hkv, D, G, n = st["T"], st["Hq"], st["Hkv"], st["D"], st["Hq"] // st["Hkv"], st["longest"]
    b, i = _tokens(st["cu"], T)
    B, S = st["after"].numel(), st["table"].shape[1] * PAGE
    q = torch.zeros((B, n, Hq, D), device=DEV)
    q[b, i] = st["q"].float()
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    page = st["table"].clamp(min=0).long()

    def values(pool, scale):
        x = pool[page] if scale is None else pool[page].view(torch.float8_e4m3fn)
        return x.float() if scale is None else x.float() * scale[page][..., None, None]

    k = values(st["kp"], st["ks"]).permute(0, 2, 4, 1, 3).reshape(B, Hkv, D, S)
    s = torch.matmul(q, k).mul_(_scale(D)).view(B, Hkv, G, n, S)
    before = (st["after"] - (st["cu"][1:] - st["cu"][:-1])).long()
    seen = torch.arange(S, device=DEV) <= (before[:, None] + torch.arange(n, device=DEV))[:, :, None]
    s = s.masked_fill_(~seen[:, None, None], float("-inf"))
    m = s.amax(dim=-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = s.sub_(m).exp_()
    z = p.sum(dim=-1, keepdim=True)
    v = values(st["vp"], st["vs"]).permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, D)
    o = torch.matmul(p.view(B, Hkv, G * n, S), v).view(B, Hkv, G, n, D) / torch.where(z > 0, z, torch.ones_like(z))
    lse = (m + z.log()).squeeze(-1)
    return {"out": o[b, :, :, i].reshape(T, Hq, D).to(torch.bfloat16), "lse": lse[b, :, :, i].reshape(T, Hq)}


# ---- one pass -----------------------------------------------------------------------------------------

def _pools(st):
    codes = st["ks"] is not None
    return {"k_pool": st["kp"].view(torch.float8_e4m3fn) if codes else st["kp"], "v_pool": st["vp"].view(torch.float8_e4m3fn) if codes else st["vp"],
            "k_scale": st["ks"], "v_scale": st["vs"]}


def run(state):
    st, kind = state, state["kind"]
    if own:
        if kind == "rotate":
            st["decoder"].rotate(st["call"])
            return {"q": st["q_out"], "k": st["k_out"]}
        if kind == "append":
            st["decoder"].append_chunk(st["call"])
            return {"q": st["q_out"], **_pools(st)}
        st["decoder"].extend(st["call"])
        return {"out": st["out"], "lse": st["lse"]}
    if kind == "extend":
        return _plain_extend(st)
    if kind == "rotate":
        positions = st["positions"]
    else:
        b, i = _tokens(st["cu"], st["T"])
        positions = st["before"][b] + i
    turn = (positions, st["rope"], st["rot"], st["interleaved"])
    q, k = _turned(st["q"].float(), st["qw"], *turn), _turned(st["k"].float(), st["kw"], *turn)
    if kind == "rotate":
        return {"q": q.to(torch.bfloat16), "k": k.to(torch.bfloat16)}
    where = (st["table"], st["before"], st["cu"], st["longest"])
    _plain_write(st["kp"], st["ks"], k, *where)
    _plain_write(st["vp"], st["vs"], st["v"].float(), *where)
    return {"q": q.to(torch.bfloat16), **_pools(st)}


# ---- the same in 64 bits ------------------------------------------------------------------------------

def _exact_rows(x, w, positions, st):
    """The formula, pair by pair: (x_a, x_b) of a row turned by the angle whose cosine and sine the table has."""
    y = x.double()
    if w is not None:
        y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + EPS) * w.double()
    half = st["rot"] // 2
    table = st["rope"].double()[positions.long()]
    z = y.clone()
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if st["interleaved"] else (j, j + half)
        c, s = table[:, j, None], table[:, half + j, None]
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., a] * s + y[..., b] * c
    return z


def _exact_pool(pool, scale, rows, st):
    """(pool, scale) after the append, page by page; what an E4M3 code stands for before it is rounded."""
    table, before, cu = (st[x].cpu().numpy() for x in ("table", "before", "cu"))
    out = pool.double() if scale is None else pool.view(torch.float8_e4m3fn).double()
    new_scale = None if scale is None else scale.double()
    for b in range(len(before)):
        t, at, end = int(cu[b]), int(before[b]), int(before[b]) + int(cu[b + 1] - cu[b])
        if scale is None and end > at:
            where = torch.arange(at, end, device=DEV)
            out[_dev(table[b]).long()[where // PAGE], :, where % PAGE] = rows[t:t + end - at]
            continue
        while at < end:
            p, slot = int(table[b, at // PAGE]), at % PAGE
            take = min(PAGE - slot, end - at)
            x = rows[t:t + take].transpose(0, 1)                    # [Hkv, take, D]
            top = x.abs().amax(dim=(1, 2))
            s = torch.where(top > 0, top / 448.0, torch.ones_like(top))
            if slot:
                was = new_scale[p].clone()
                s = torch.where(top <= was * 448.0, was, s)
                out[p, :, :slot] *= (was / s)[:, None, None]
            out[p, :, slot:slot + take] = x / s[:, None, None]
            new_scale[p] = s
            at, t = at + take, t + take
    return out, new_scale


def _exact_attention(q, k, v, scale, before):
    """q [n, Hq, D] over k, v [S, Hkv, D] in 64 bits: token i sees the first before + i + 1 keys.  (out, lse)"""
    n, Hq, D = q.shape
    S, Hkv, G = k.shape[0], k.shape[1], Hq // k.shape[1]
    out, lse = torch.empty_like(q), torch.empty((n, Hq), dtype=q.dtype, device=q.device)
    hidden = torch.arange(S, device=DEV)[None, :] > before + torch.arange(n, device=DEV)[:, None]
    for h in range(Hkv):
        kt, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
        for g in range(G):
            s = (q[:, h * G + g].contiguous() @ kt).mul_(scale).masked_fill_(hidden, float("-inf"))
            top = s.amax(dim=-1, keepdim=True)
            w = s.sub_(top).exp_()
            z = w.sum(dim=-1, keepdim=True)
            out[:, h * G + g], lse[:, h * G + g] = (w @ vh) / z, (top + z.log()).squeeze(-1)
    return out, lse


def exact(case, seed):
    st = prepare(case, seed)
    if st["kind"] == "rotate":
        return {"q": _exact_rows(st["q"], st["qw"], st["positions"], st), "k": _exact_rows(st["k"], st["kw"], st["positions"], st)}
    cu = st["cu"].cpu().tolist()
    if st["kind"] == "append":
        positions = torch.cat([int(x) + torch.arange(m - l, device=DEV) for x, l, m in zip(st["before"].cpu(), cu, cu[1:])])
        kp, ks = _exact_pool(st["kp"], st["ks"], _exact_rows(st["k"], st["kw"], positions, st), st)
        vp, vs = _exact_pool(st["vp"], st["vs"], st["v"].double(), st)
        return {"q": _exact_rows(st["q"], st["qw"], positions, st), "k_pool": kp, "v_pool": vp, "k_scale": ks, "v_scale": vs}
    out, lse = (torch.empty(st[x].shape, dtype=torch.float64, device=DEV) for x in ("out", "lse"))
    for b, L in enumerate(st["after"].cpu().tolist()):
        n = cu[b + 1] - cu[b]
        if not n:
            continue
        ids = st["table"][b, :_pages(L)].long()

        def tokens(pool, scale):
            x = pool[ids].double() if scale is None else pool[ids].view(torch.float8_e4m3fn).double() * scale[ids].double()[:, :, None, None]
            return x.transpose(1, 2).reshape(-1, st["Hkv"], st["D"])[:L]

        at = slice(cu[b], cu[b + 1])
        out[at], lse[at] = _exact_attention(st["q"][at].double(), tokens(st["kp"], st["ks"]), tokens(st["vp"], st["vs"]), _scale(st["D"]), L - n)
    return {"out": out, "lse": lse}
