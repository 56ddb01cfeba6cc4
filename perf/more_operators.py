"""Measured cases of the operators at both ends of a serving step over a paged cache, and their plain forms.

Before the layers, every new token of every sequence needs a page and a slot: lengths live on the GPU, so block tables, packed
offsets, positions and slots are built there, from a stack of free pages.  After the layers, the drafted tokens that a step has
looked at are verified against the target's probabilities, and each sequence gets its next token; sequences that end give their
pages back.

  place    pages and slots for the new tokens of a batch: rows of the block table grown, cu_seqlens, positions, slots
  release  pages that the sequences no longer need, back to the stack
  verify   speculative sampling: drafts accepted in order against softmax(logits / temperature), and a token drawn by one given
           random number from what is left; one row a sequence is the choice of the next token

Batches and lengths are those of this repository's workloads (workload/gen.py: 256 sequences in groups of eight over a shared
prompt, 512 ... 4096 tokens) and generic ones beside them; vocabularies are generic.  Lengths belong to the case (they come from
its "length_seed"); values, page placement and random numbers come from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda:0"

_decoder = None


def decoder():
    """The process's one decoder (a context and its workspace), as a worker keeps it."""
    global _decoder
    if _decoder is None:
        import paper_2507_01663_amd as ra
        _decoder = ra.Decoder(0)
    return _decoder


# ---- the cases ----------------------------------------------------------------------------------------

def _pages_case(name, kind, seqs, new, context, group=0, prefix=0, tight=False, length_seed=0):
    """new: (least, most) new tokens (place) or tokens kept of the context (release, where some sequences keep all of them);
    context: tokens held before; group: sequences that share `prefix` pages (0: none do); tight: the stack does not hold what
    the batch asks for."""
    return {"name": name, "kind": kind, "seqs": seqs, "new_lo": new[0], "new_hi": new[1], "context_lo": context[0], "context_hi": context[1],
            "group": group, "prefix": prefix, "tight": tight, "length_seed": length_seed}


def _verify_case(name, seqs, rows, vocab, dtype="bf16", drafts="logits", temperature="one", pad=0, length_seed=0):
    """rows: (least, most) rows of logits of a sequence, one more than its drafts; drafts: whether the draft model's logits come with
    them ("logits") or the drafts are plain guesses ("guess"); temperature: 1 for all, or of each sequence's own, zeros among them
    ("mixed"); pad: elements between two rows."""
    return {"name": name, "kind": "verify", "seqs": seqs, "rows_lo": rows[0], "rows_hi": rows[1], "vocab": vocab, "dtype": dtype, "drafts": drafts,
            "temperature": temperature, "pad": pad, "length_seed": length_seed}


def listed():
    return [
        # the next token of every sequence of the 7B-shaped batch: eight responses to a prompt, one page in sixteen is full
        _pages_case("place_step", "place", 256, (1, 1), (512, 4095), group=8, prefix=32),
        # the turns of a batch, ragged, with sequences that wait; the stack runs dry before the last ones
        _pages_case("place_turns_tight", "place", 777, (0, 190), (1, 900), tight=True),
        # many long prompts at once
        _pages_case("place_prompts", "place", 512, (30, 2000), (0, 0)),
        # a few responses have ended, and drafts that were turned down leave a page here and there
        _pages_case("release_ended", "release", 256, (0, 600), (512, 4096), group=8, prefix=32),
        # the end of a batch: everything comes back
        _pages_case("release_all", "release", 2048, (0, 0), (1024, 17408)),
        # the next token of a handful of sequences, a call that is all latency
        _verify_case("next_token_few", 4, (1, 1), 32000),
        # the next token of every sequence of a batch, some greedy and some not
        _verify_case("next_token_batch", 256, (1, 1), 152064, temperature="mixed"),
        # a draft of four tokens for one sequence: an interactive session
        _verify_case("drafts_one", 1, (5, 5), 128256),
        # drafts of four tokens for every sequence of a batch, with the draft model's logits
        _verify_case("drafts_batch", 128, (5, 5), 152064),
        # guesses from the text so far, ragged, rows of an odd length in a padded tensor, float32
        _verify_case("guesses_ragged_fp32", 96, (1, 9), 50257, dtype="fp32", drafts="guess", temperature="mixed", pad=47),
        # the largest: float32 logits of a batch of drafts
        _verify_case("drafts_batch_fp32", 200, (4, 6), 152064, dtype="fp32"),
    ]


MOST_VALUES = 1.5e8          # logits of a drawn case, target's and draft's together


def _spread(rng, lo, hi):
    """An integer of lo .. hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["place", "place", "release", "verify", "verify", "verify", "verify"])
    while True:
        seed = rng.randrange(1 << 30)
        if kind == "verify":
            most = _spread(rng, 1, 12)
            c = _verify_case("", _spread(rng, 1, 400), (rng.choice([1, most, rng.randint(1, most)]), most), _spread(rng, 500, 160000), rng.choice(["bf16", "fp32"]),
                             rng.choice(["logits", "logits", "guess"]), rng.choice(["one", "mixed"]), rng.choice([0, 0, rng.randint(1, 64)]), seed)
            ok = 2 * c["seqs"] * most * c["vocab"] <= MOST_VALUES
        else:
            deep, grouped = _spread(rng, 1, 17000), rng.random() < 0.4
            most = _spread(rng, 1, 2000)
            c = _pages_case("", kind, _spread(rng, 1, 2000), (rng.choice([0, 1, most]) if most > 0 else 0, most), (deep // rng.choice([1, 2, 4]), deep),
                            rng.randint(2, 16) if grouped else 0, rng.randint(1, 40) if grouped else 0, kind == "place" and rng.random() < 0.3, seed)
            ok = c["seqs"] * (deep + most) <= 1.6e7 and c["seqs"] * most <= 6e5 and work(c)["flops"] > 0
        if ok:
            del c["name"]
            return c


# ---- lengths ------------------------------------------------------------------------------------------

def _rows(case):
    r = random.Random(case["length_seed"])
    return [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["seqs"])]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _lengths(case):
    """(new tokens or tokens kept, tokens held, pages held, shared pages) of every sequence; a group's sequences follow each other."""
    r, n = random.Random(case["length_seed"]), case["seqs"]
    shared = case["prefix"] if case["group"] else 0
    held = [max(r.randint(case["context_lo"], case["context_hi"]), shared * PAGE) for _ in range(n)]
    if case["kind"] == "place":
        new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(n)]
        # a page to spare here and there: what drafts that were turned down have left; a group's new sequences hold nothing of their own yet
        pages = [0 if shared and h == shared * PAGE else _pages(h) + (r.random() < 0.2) for h in held]
    else:
        new = [min(h, r.randint(case["new_lo"], case["new_hi"])) if case["new_hi"] == 0 or r.random() < 0.25 else max(0, h - r.randint(0, 8)) for h in held]
        pages = [_pages(h) for h in held]
    return new, held, pages, shared


def _supply(case):
    """Pages on the stack before the call."""
    new, held, pages, shared = _lengths(case)
    if case["kind"] == "release":
        return 100
    need = sum(max(0, _pages(a + b) - max(p, shared)) for a, b, p in zip(new, held, pages) if a)
    return need * 9 // 10 if case["tight"] else need + 50


# ---- what the path cannot do without ------------------------------------------------------------------

def work(case):
    if case["kind"] == "verify":
        rows, e = _rows(case), 2 if case["dtype"] == "bf16" else 4
        drafted = sum(rows) - len(rows) if case["drafts"] == "logits" else 0
        values = (sum(rows) + drafted) * case["vocab"]
        return {"bytes": values * e + 16 * sum(rows) + 16 * len(rows), "flops": 4 * values}
    new, held, pages, shared = _lengths(case)
    n = case["seqs"]
    if case["kind"] == "place":
        tokens, taken = sum(new), min(_supply(case), sum(max(0, _pages(a + b) - max(p, shared)) for a, b, p in zip(new, held, pages) if a))
        return {"bytes": 24 * n + 8 * taken + 16 * tokens, "flops": 4 * tokens}
    back = sum(max(0, p - max(_pages(k), shared)) for k, p in zip(new, pages))
    return {"bytes": 12 * n + 8 * back, "flops": back}


# ---- inputs -------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _ints(x):
    return _dev(np.asarray(x, dtype=np.int32))


def _logits(rows, vocab, pad, dtype, g):
    """Logits as a head gives them: most tokens unlikely, a few that carry the row."""
    x = torch.empty((rows, vocab + pad), dtype=torch.float32, device=DEV)
    for a in range(0, rows, 256):
        x[a:a + 256].normal_(0.0, 2.0, generator=g)
    some = torch.randint(vocab, (rows, 24), generator=g, device=DEV)
    x.scatter_add_(1, some, torch.empty(some.shape, device=DEV).exponential_(0.2, generator=g) + 4.0)
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def _sample(logits, temperature, g):
    """A token of each row, by the largest of perturbed logits."""
    out = torch.empty(logits.shape[0], dtype=torch.int32, device=DEV)
    for a in range(0, logits.shape[0], 256):
        x = logits[a:a + 256].float() / temperature[a:a + 256, None].clamp(min=0.05)
        x -= torch.empty_like(x).exponential_(generator=g).log_()
        out[a:a + 256] = x.argmax(dim=-1).to(torch.int32)
    return out


def _prepare_verify(case, seed):
    g = _generator(seed)
    rows, V = np.array(_rows(case), dtype=np.int64), case["vocab"]
    B, R = len(rows), int(rows.sum())
    cu = np.concatenate([[0], np.cumsum(rows)])
    owner = np.repeat(np.arange(B), rows)
    last = np.zeros(R, dtype=bool)
    last[cu[1:] - 1] = True
    judging = _dev(np.flatnonzero(~last))                    # rows that judge a draft, in order: row i is a draft's i-th
    st = {"kind": "verify", "B": B, "R": R, "V": V, "cu": _ints(cu), "owner": _dev(owner), "judging": judging, "longest": int(rows.max())}
    full = _logits(R, V, case["pad"], case["dtype"], g)
    st["logits"] = full[:, :V]
    T = torch.ones(B, device=DEV)
    if case["temperature"] == "mixed":
        T = (0.3 + torch.rand(B, generator=g, device=DEV)) * (torch.rand(B, generator=g, device=DEV) > 0.25)
    st["temperature"] = T
    st["tokens"] = torch.randint(V, (R,), generator=g, device=DEV, dtype=torch.int32)
    st["draft_logits"] = st["draft_rows"] = None
    if judging.numel():
        if case["drafts"] == "logits":                       # a draft model that is mostly of the target's mind
            d = torch.empty((judging.numel(), V + case["pad"]), dtype=full.dtype, device=DEV)
            for a in range(0, judging.numel(), 256):
                x = full[judging[a:a + 256]].float()
                d[a:a + 256] = x + torch.empty_like(x).normal_(0.0, 0.7, generator=g)
            st["draft_logits"], st["draft_rows"] = d[:, :V], _ints(cu[:-1] - np.arange(B))
            st["tokens"][judging + 1] = _sample(st["draft_logits"], T[st["owner"][judging]], g)
        else:                                                # text that repeats itself: a guess that is often right
            right = torch.rand(judging.numel(), generator=g, device=DEV) < 0.6
            good = _sample(st["logits"][judging], T[st["owner"][judging]], g)
            st["tokens"][judging + 1] = torch.where(right, good, st["tokens"][judging + 1])
    st["u"], st["v"] = torch.rand(R, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    st["accepted"], st["next"] = (torch.empty(B, dtype=torch.int32, device=DEV) for _ in range(2))
    st["out"], st["logprobs"] = torch.empty(R, dtype=torch.int32, device=DEV), torch.empty(R, device=DEV)
    return st


def _prepare_pages(case, seed):
    g = _generator(seed)
    new, held, pages, shared = _lengths(case)
    B, supply, kind = case["seqs"], _supply(case), case["kind"]
    groups = (B + case["group"] - 1) // case["group"] if shared else 0
    most = max(max(_pages(a + b) if kind == "place" else _pages(b) for a, b in zip(new, held)), max(pages), shared)
    mine = [max(0, p - shared) for p in pages]
    num_pages = max(1, sum(mine) + supply + groups * shared + 7)
    ids = torch.randperm(num_pages, generator=g, device=DEV).to(torch.int32).cpu().numpy()
    table = np.full((B, most), -1, dtype=np.int32)
    prefix = ids[:groups * shared].reshape(groups, -1) if shared else None
    at = groups * shared
    for b in range(B):
        if shared and pages[b]:
            table[b, :shared] = prefix[b // case["group"]]
        table[b, shared:shared + mine[b]] = ids[at:at + mine[b]]
        at += mine[b]
    stack = np.full(num_pages, -1, dtype=np.int32)
    stack[:supply] = ids[at:at + supply]
    st = {"kind": kind, "B": B, "num_pages": num_pages, "table": _dev(table), "lens": _ints(held), "held": _ints(pages), "asked": _ints(new),
          "stack": _dev(stack), "free": _ints([supply]), "held_out": torch.empty(B, dtype=torch.int32, device=DEV),
          "free_out": torch.empty(1, dtype=torch.int32, device=DEV), "group": None, "offsets": None, "prefix": None, "T": sum(new)}
    if shared:
        st["group"], st["offsets"] = _ints(np.arange(B) // case["group"]), _ints(np.arange(groups + 1) * shared)
        st["prefix"] = _dev(prefix.reshape(-1))
    if kind == "place":
        st["cu"], st["after"] = torch.empty(B + 1, dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)
        st["positions"], st["seqs"] = (torch.empty(st["T"], dtype=torch.int32, device=DEV) for _ in range(2))
        st["slots"] = torch.empty(st["T"], dtype=torch.int64, device=DEV)
    return st


def prepare(case, seed):
    st = _prepare_verify(case, seed) if case["kind"] == "verify" else _prepare_pages(case, seed)
    if own:         # the call's descriptor: addresses and sizes, which a worker fills in once for its buffers
        import paper_2507_01663_amd as ra
        st["decoder"] = decoder()
        if st["kind"] == "verify":
            st["call"] = ra.verify_from_tensors(st["logits"], st["cu"], st["tokens"], st["u"], st["v"], st["accepted"], st["out"], st["logprobs"],
                                                st["next"], temperature=st["temperature"], draft_logits=st["draft_logits"], draft_rows=st["draft_rows"])
        elif st["kind"] == "place":
            st["call"] = ra.place_from_tensors(st["lens"], st["asked"], st["held"], st["table"], st["stack"], st["free"], st["cu"], st["after"],
                                               st["held_out"], st["free_out"], positions=st["positions"], slots=st["slots"], seqs=st["seqs"],
                                               seq_group=st["group"], prefix_page_offsets=st["offsets"], prefix_pages=st["prefix"])
        else:
            st["call"] = ra.release_from_tensors(st["asked"], st["held"], st["table"], st["stack"], st["free"], st["held_out"], st["free_out"],
                                                 seq_group=st["group"], prefix_page_offsets=st["offsets"])
    return st


# ---- the plain forms ----------------------------------------------------------------------------------

def _shared(st):
    """Shared pages of each sequence."""
    if st["group"] is None:
        return torch.zeros(st["B"], dtype=torch.int64, device=DEV)
    return (st["offsets"][1:] - st["offsets"][:-1]).long()[st["group"].long()]


def _plain_place(st):
    table, M, T = st["table"], st["table"].shape[1], st["T"]
    L, n, H, free, F = st["lens"].long(), st["asked"].long(), st["held"].long(), st["free"].long(), _shared(st)
    S, P = torch.maximum(H, F), (L + n + PAGE - 1) // PAGE
    fine = (n > 0) & (L <= PAGE * S) & (P <= M)
    need, n = torch.where(fine, (P - S).clamp(min=0), 0), torch.where(fine, n, 0)
    served = fine & ((need == 0) | (need.cumsum(0) <= free)) & (n.cumsum(0) <= T)
    need, n = torch.where(served, need, 0), torch.where(served, n, 0)
    i = torch.arange(M, device=DEV)
    if st["group"] is not None:
        copied = served[:, None] & (i >= H[:, None]) & (i < F[:, None])
        source = (st["offsets"].long()[st["group"].long()][:, None] + i).clamp(max=st["prefix"].numel() - 1)
        table.copy_(torch.where(copied, st["prefix"][source], table))
    taken = served[:, None] & (i >= S[:, None]) & (i < P[:, None])
    source = free - 1 - (need.cumsum(0) - need)[:, None] - (i - S[:, None])
    table.copy_(torch.where(taken, st["stack"][source.clamp(0, st["num_pages"] - 1)], table))
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), n.cumsum(0)])
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=st["B"] - 1)
    there = t < cu[-1]
    position = torch.where(there, L[b] + t - cu[b], 0)
    slot = table[b, (position // PAGE).clamp(max=M - 1)].long() * PAGE + position % PAGE
    return {"table": table, "held": torch.where(served, torch.maximum(S, P), H).int(), "free": (free - need.sum()).int(), "after": (L + n).int(),
            "cu": cu.int(), "positions": torch.where(there, position, -1).int(), "slots": torch.where(there, slot, -1),
            "seqs": torch.where(there, b, -1).int()}


def _plain_release(st):
    table, M, stack = st["table"], st["table"].shape[1], st["stack"]
    H, free = st["held"].long(), st["free"].long()
    K = torch.minimum((st["asked"].long() + PAGE - 1) // PAGE, H)
    begin = torch.maximum(K, _shared(st))
    back = (H - begin).clamp(min=0)
    i = torch.arange(M, device=DEV)
    given = (i >= begin[:, None]) & (i < H[:, None])
    to = free + (back.cumsum(0) - back)[:, None] + (i - begin[:, None])
    stack[to[given]] = table[given]
    return {"held": K.int(), "stack": stack, "free": (free + back.sum()).int()}


def _probabilities(x, T):
    """softmax(x / T) of each row in 64 bits; where T is 0, all of it on the first of the largest."""
    x = x.double()
    e = ((x - x.amax(dim=-1, keepdim=True)) / torch.where(T > 0, T, 1.0).double()[:, None]).exp_()
    e /= e.sum(dim=-1, keepdim=True)
    sure = torch.arange(x.shape[1], device=DEV) == x.argmax(dim=-1, keepdim=True)
    return torch.where((T > 0)[:, None], e, sure.double())


def _plain_verify(st):
    B, R, V, cu, judging, owner = st["B"], st["R"], st["V"], st["cu"].long(), st["judging"], st["owner"]
    T = st["temperature"]
    p = _probabilities(st["logits"], T[owner])
    drafted = st["tokens"].long()[judging + 1]
    accepted = torch.zeros(B, dtype=torch.int64, device=DEV)
    at = cu[:-1]
    if judging.numel():
        chance = p[judging, drafted]
        if st["draft_logits"] is not None:
            q = _probabilities(st["draft_logits"], T[owner[judging]])
            passed = st["u"].double()[judging] * q[torch.arange(judging.numel(), device=DEV), drafted] < chance
        else:
            passed = st["u"].double()[judging] < chance
        run = torch.zeros((B, st["longest"]), dtype=torch.int64, device=DEV)
        run[owner[judging], judging - cu[owner[judging]]] = passed.long()
        accepted = run.cumprod(dim=1).sum(dim=1)
        at = cu[:-1] + accepted
    w = p[at]
    if judging.numel():
        b = torch.nonzero(at < cu[1:] - 1).squeeze(1)        # sequences with a draft that was turned down
        if st["draft_logits"] is not None:
            left = (w[b] - q[at[b] - b]).clamp(min=0)        # (a draft's rows: one fewer for every sequence before)
        else:
            left = w[b]
            left[torch.arange(b.numel(), device=DEV), st["tokens"].long()[at[b] + 1]] = 0
        w[b] = torch.where(left.sum(dim=1, keepdim=True) > 0, left, w[b])
    c = w.cumsum(dim=1)
    some = torch.arange(V, device=DEV) * (w > 0)
    token = torch.minimum((c <= st["v"].double()[:, None] * c[:, -1:]).sum(dim=1), some.amax(dim=1))
    place = torch.arange(R, device=DEV) - cu[owner]
    following = torch.cat([st["tokens"].long()[1:], torch.zeros(1, dtype=torch.int64, device=DEV)])
    out = torch.where(place < accepted[owner], following, torch.where(place == accepted[owner], token[owner], -1))
    lp = p.gather(1, out.clamp(min=0)[:, None]).squeeze(1).log()
    return {"accepted": accepted.int(), "tokens": out.int(), "logprobs": torch.where(out >= 0, lp, 0.0).float(), "next": token.int()}


# ---- one pass -----------------------------------------------------------------------------------------

def run(state):
    st, kind = state, state["kind"]
    if own:
        if kind == "verify":
            st["decoder"].verify(st["call"])
            return {"accepted": st["accepted"], "tokens": st["out"], "logprobs": st["logprobs"], "next": st["next"]}
        if kind == "place":
            st["decoder"].place(st["call"])
            return {"table": st["table"], "held": st["held_out"], "free": st["free_out"], "after": st["after"], "cu": st["cu"],
                    "positions": st["positions"], "slots": st["slots"], "seqs": st["seqs"]}
        st["decoder"].release(st["call"])
        return {"held": st["held_out"], "stack": st["stack"], "free": st["free_out"]}
    return _plain_verify(st) if kind == "verify" else _plain_place(st) if kind == "place" else _plain_release(st)


# ---- the same from the definition ---------------------------------------------------------------------

def _exact_place(st):
    table, stack = st["table"].cpu().numpy().copy(), st["stack"].cpu().numpy()
    lens, asked, held = (st[x].cpu().numpy().astype(np.int64) for x in ("lens", "asked", "held"))
    held_out, after, cu = held.copy(), lens.copy(), [0]
    top = free = int(st["free"][0])
    wanted = tokens = 0                                      # what the sequences so far would like to have
    positions, slots, seqs = [], [], []
    for b in range(st["B"]):
        n, H, row = int(asked[b]), int(held[b]), table[b]
        group = None if st["group"] is None else int(st["group"][b])
        shared = [] if group is None else st["prefix"][int(st["offsets"][group]):int(st["offsets"][group + 1])].cpu().numpy()
        end = int(lens[b]) + n
        pages = max(H, len(shared))
        if n > 0 and lens[b] <= PAGE * pages and _pages(end) <= table.shape[1]:
            extra = max(0, _pages(end) - pages)
            wanted, tokens = wanted + extra, tokens + n
            if (not extra or wanted <= free) and tokens <= st["T"]:
                for j in range(H, len(shared)):
                    row[j] = shared[j]
                for j in range(pages, pages + extra):
                    top -= 1
                    row[j] = stack[top]
                held_out[b], after[b] = pages + extra, end
                where = np.arange(lens[b], end)
                positions.append(where), slots.append(row[where // PAGE].astype(np.int64) * PAGE + where % PAGE), seqs.append(np.full(n, b))
        cu.append(int(after[:b + 1].sum() - lens[:b + 1].sum()))

    def packed(x):
        x = np.concatenate(x) if x else np.zeros(0, dtype=np.int64)
        return np.concatenate([x, np.full(st["T"] - len(x), -1)])

    return {"table": _dev(table), "held": _ints(held_out), "free": _ints([top]), "after": _ints(after), "cu": _ints(cu),
            "positions": _ints(packed(positions)), "slots": _dev(packed(slots).astype(np.int64)), "seqs": _ints(packed(seqs))}


def _exact_release(st):
    table, stack = st["table"].cpu().numpy(), st["stack"].cpu().numpy().copy()
    keep, held = st["asked"].cpu().numpy(), st["held"].cpu().numpy().copy()
    top = int(st["free"][0])
    for b in range(st["B"]):
        group = None if st["group"] is None else int(st["group"][b])
        shared = 0 if group is None else int(st["offsets"][group + 1]) - int(st["offsets"][group])
        kept = min(_pages(int(keep[b])), int(held[b]))
        for j in range(max(kept, shared), int(held[b])):
            stack[top] = table[b, j]
            top += 1
        held[b] = kept
    return {"held": _ints(held), "stack": _dev(stack), "free": _ints([top])}


def _exact_row(x, T):
    x = x.double()
    if T == 0:
        p = torch.zeros_like(x)
        p[torch.nonzero(x == x.max())[0]] = 1.0
        return p
    return torch.exp(x / T - torch.logsumexp(x / T, dim=0))


def _exact_verify(st):
    cu, tokens, V = st["cu"].tolist(), st["tokens"].tolist(), st["V"]
    u, v, T = st["u"].double().tolist(), st["v"].double().tolist(), st["temperature"].double().tolist()
    accepted, following = [], []
    out, logprobs = torch.full((st["R"],), -1, dtype=torch.int32), torch.zeros(st["R"], dtype=torch.float64)
    for b, (first, end) in enumerate(zip(cu, cu[1:])):
        for t in range(first, end):
            p = _exact_row(st["logits"][t], T[b])
            w = p
            if t < end - 1:
                x = tokens[t + 1]
                q = torch.zeros_like(p)
                if st["draft_logits"] is None:
                    q[x] = 1.0
                else:
                    q = _exact_row(st["draft_logits"][t - b], T[b])
                if u[t] * float(q[x]) < float(p[x]):
                    out[t], logprobs[t] = x, math.log(float(p[x]))
                    continue
                w = torch.relu(p - q)
                if float(w.sum()) <= 0:
                    w = p
            # the first token at which the sum of all up to it exceeds its share of the whole
            c = torch.cumsum(w, dim=0)
            x = min(int(torch.searchsorted(c, v[b] * c[-1], right=True)), int(torch.nonzero(w)[-1]))
            out[t], logprobs[t] = x, math.log(float(p[x]))
            accepted.append(t - first), following.append(x)
            break
    return {"accepted": _ints(accepted), "tokens": out.to(DEV), "logprobs": logprobs.to(DEV), "next": _ints(following)}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_verify(st) if st["kind"] == "verify" else _exact_place(st) if st["kind"] == "place" else _exact_release(st)
