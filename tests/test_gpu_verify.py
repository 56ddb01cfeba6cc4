"""Verification of drafts and the choice of next tokens, on the GPU, against the plain form in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2507_01663_amd as ra
from gpu_util import context
from step_util import DEV, Verifying, distribution, drafting, rounded, rows_of

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", params=["binary64 sums", "binary32 sums first"])
def dec(request):
    """The library's choice for the few logits of most of these tests, and the way that it takes with many."""
    exact = request.param == "binary64 sums"
    d = context() if exact else context(VERIFY_FEW=0)
    d.exact = exact
    yield d
    d.close()


def run(dec, x, what=""):
    x.exact = dec.exact
    dec.verify(x.c)
    return x.check(what)


VOCABS = [1, 2, 7, 8, 9, 63, 300, 2047, 2048, 2049, 4099, 16384, 16385, 50257]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_drafts(dec, V, dtype):
    """Ragged rows, sequences without any among them, with and without the draft model's logits, own temperatures with zeros among
    them; rows aligned and not, with gaps; rows of nobody before and behind."""
    rows = [3, 0, 1, 5, 2, 0, 0, 4, 1] if V < 20000 else [3, 0, 2]
    T = [1.0, 0.5, 0.0, 1.7, 0.3, 1.0, 1.0, 0.0, 1e-3][:len(rows)]
    for seed, (drafts, temper, pad, shift, lead, behind) in enumerate([("logits", None, 0, 0, 0, 0), ("logits", T, 3, 1, 2, 3), ("guess", None, 1, 0, 0, 2),
                                                                       ("guess", T, 0, 5, 1, 0), ("logits", T, 8, 8, 0, 0)]):
        print("case V", V, dtype, drafts, temper is not None, pad, shift, flush=True)
        run(dec, drafting(7 * V + seed, rows, V, dtype, drafts, temper, pad=pad, shift=shift, lead=lead, behind=behind), (V, dtype, seed))


@pytest.mark.parametrize("dtype,draft_dtype", [("bf16", "fp32"), ("fp32", "bf16")])
def test_a_draft_model_of_another_type(dec, dtype, draft_dtype):
    run(dec, drafting(3, [4, 3, 1, 6], 3001, dtype, draft_dtype=draft_dtype))


@pytest.mark.parametrize("V", [5, 2048, 30000])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_next_tokens(dec, V, dtype):
    """One row a sequence: the choice of the next token, at many numbers."""
    n = 200 if V < 10000 else 40
    T = np.where(np.arange(n) % 5 == 0, 0.0, 0.2 + np.arange(n) % 7 / 4)
    for temper in (None, T):
        run(dec, drafting(V, [1] * n, V, dtype, "guess", temper))


@pytest.mark.parametrize("rows,V", [(1, 152064), (5, 128256), (2, 100003)])
def test_few_long_rows(dec, rows, V):
    for drafts in ("logits", "guess"):
        run(dec, drafting(rows, [rows, 1], V, "bf16", drafts))


@pytest.mark.parametrize("drafts", ["logits", "guess"])
def test_rows_of_more_parts_than_a_wave_has_lanes(dec, drafts):
    """More than 64 parts of 4096 values to a row; of the flat ones no binary32 sum settles anything."""
    x = drafting(5, [2, 3, 1], 300001, "bf16", drafts, [1.0, 0.0, 2.5])
    run(dec, x)
    flat = rows_of(6, 60, 300001, "fp32", 0.1) if drafts == "guess" else rows_of(6, 4, 540000, "fp32", 0.1)
    n = len(flat) // 2
    r = np.random.default_rng(7)
    x = Verifying([2] * n, flat, r.integers(0, flat.shape[1], 2 * n), np.full(2 * n, 0.5), r.random(n), draft=None if drafts == "guess" else flat[::-1][:n].copy(),
                  draft_rows=None if drafts == "guess" else list(range(n)), dtype="fp32")
    run(dec, x)


@pytest.mark.parametrize("n", [63, 64, 65, 130])
@pytest.mark.parametrize("V", [40, 9000])
def test_many_sequences(dec, n, V):
    """As many sequences as a wave has lanes, and one more; as many rows each, ragged ones, none for the first and the last; rows of
    nobody before and behind."""
    T = np.where(np.arange(n) % 6 == 1, 0.0, 0.3 + np.arange(n) % 4 / 3)
    for seed, rows in enumerate([[2] * n, [0] + [1 + b % 3 for b in range(n - 2)] + [0], [b % 2 * 3 for b in range(n)]]):
        for drafts in ("logits", "guess"):
            run(dec, drafting(n + seed, rows, V, "bf16", drafts, T if seed else None, lead=seed, behind=2 * seed), (n, V, seed, drafts))


@pytest.mark.parametrize("rows", [20, 70, 200])
def test_long_drafts(dec, rows):
    """More rows than a workgroup looks at together; drafts that all stay."""
    r = np.random.default_rng(rows)
    logits = rows_of(rows, rows + 3, 50, "fp32")
    tokens = r.integers(0, 50, rows + 3)
    u = np.zeros(rows + 3)
    run(dec, Verifying([rows, 3], logits, tokens, u, [0.3, 0.9], dtype="fp32"))
    u[rows - 5] = 1.0
    run(dec, Verifying([rows, 3], logits, tokens, u, [0.3, 0.9], draft=logits, draft_rows=[0, rows], dtype="fp32"))
    run(dec, Verifying([rows, 3], logits, tokens, u, [0.3, 0.9], draft=rounded(logits + 1.0, "fp32"), draft_rows=[0, rows], dtype="fp32"))


def test_a_draft_model_like_the_target(dec):
    """The same logits on both sides: every draft stays at every number below one, and what is drawn behind a draft that a number of
    one turned down is drawn from the target (nothing is left of p - q)."""
    logits = rows_of(4, 5, 4000, "fp32")
    tokens = [0, 17, 1999, 3, 3999]
    for below in (0.0, 0.5, float(np.float32(1 - 2.0 ** -24))):
        x = run(dec, Verifying([5], logits, tokens, [below] * 5, [0.4], draft=logits[:4], draft_rows=[0], dtype="fp32"))
        assert x.accepted.tolist() == [4]
    x = run(dec, Verifying([5], logits, tokens, [0.5, 1.0, 0, 0, 0], [0.4], draft=logits[:4], draft_rows=[0], dtype="fp32"))
    assert x.accepted.tolist() == [1]


@pytest.mark.parametrize("V", [40, 5000, 30000])
@pytest.mark.parametrize("pairs", [1, 7])
def test_models_that_agree_but_for_a_few_tokens(dec, V, pairs):
    """The draft's logits are the target's with a few pairs of tokens changed about: p and q are the same everywhere else, to the last
    bits, and all that is left of p - q lies in those tokens, also for numbers next to their borders (by much more than what 64-bit sums of
    one row in two orders may differ by, 1e-13 of what is left)."""
    r = np.random.default_rng(V + pairs)
    v = [0.5, 1e-6, 1 - 2.0 ** -20, 0.25, 0.75, 1e-9, float(np.float32(1 - 2.0 ** -24)), 0.01]
    n = len(v)
    logits = rows_of(V, 2 * n, V, "fp32", 1.0)
    draft = logits[::2].copy()
    tokens, starts = np.zeros(2 * n, dtype=np.int64), np.arange(n)
    for b in range(n):
        at = r.permutation(V)[:2 * pairs].reshape(pairs, 2)
        for i, j in at:
            logits[2 * b, i], logits[2 * b, j] = 4.0, 1.0
            draft[b, i], draft[b, j] = 1.0, 4.0
        tokens[2 * b + 1] = at[0, 1]                         # of the draft's liking: turned down at 0.5 of 1 / e^3
    x = run(dec, Verifying([2] * n, logits, tokens, [0.5] * (2 * n), v, draft=draft, draft_rows=starts, dtype="fp32"))
    assert x.accepted.tolist() == [0] * n
    T = [0.7, 1.3, 2.0, 0.5, 1.0, 1.0, 3.0, 0.9]
    run(dec, Verifying([2] * n, logits, tokens, [0.9] * (2 * n), v, T, draft=draft, draft_rows=starts, dtype="fp32"))


@pytest.mark.parametrize("V", [1, 4, 256, 4096, 65536])
def test_equal_logits_and_numbers_on_the_borders(dec, V):
    """V equal logits, V a power of two: every weight and sum is exact, and a number of exactly i / V draws token i."""
    at = sorted({0, 1, V // 3, V // 2, V - 1, V // 4096 * 7} & set(range(V)))
    n = len(at)
    for level, T in ((0.0, None), (-3.5, [0.25] * n), (1000.0, [2.0] * n)):
        x = Verifying([1] * n, np.full((n, V), level), [0] * n, [0.0] * n, [i / V for i in at], T)
        run(dec, x)
        assert x.next.tolist() == at
    # a guess of probability 1 / V stays at every number below that, and not at it
    for u, stays in ((1 / V, 0), (float(np.nextafter(np.float32(1 / V), np.float32(0))), 1)):
        x = run(dec, Verifying([2], np.zeros((2, V)), [0, V // 2], [u, 0], [0.5]))
        assert x.accepted.tolist() == [stays]


def test_numbers_at_and_past_their_ends(dec):
    n, V = 9, 700
    logits = rows_of(1, 2 * n, V, "fp32")
    logits[:, :3] = -INF                                     # (what a number of 0 must not draw)
    logits[:, -2:] = -INF                                    # (nor one of 1)
    v = [0.0, 1.0, -0.5, 1.5, NAN, INF, -INF, 1e-30, float(np.float32(1 - 2.0 ** -24))]
    u = [0.0, 0, 1.0, 0, -1.0, 0, 2.0, 0, NAN, 0, INF, 0, -INF, 0, 0.5, 0, 1e-40, 0]
    tokens = list(range(10, 10 + 2 * n))
    for draft in (None, rows_of(2, n, V, "fp32")):
        run(dec, Verifying([2] * n, logits, tokens, u, v, draft=draft, draft_rows=None if draft is None else list(range(n)), dtype="fp32"))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_masks(dec, dtype):
    """Logits masked by -inf or by the type's lowest value, in whole stretches, at the ends, all but one; rows that have no
    distribution: all of them -inf, a NaN, +inf.  As targets and as drafts."""
    V = 5000
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    base = rows_of(8, 1, V, dtype)[0]
    rows = []
    for mask in (-INF, low):
        for cut in (slice(0, 2500), slice(100, V), slice(0, V - 1), slice(1, V), slice(2048, 4096)):
            x = base.copy()
            x[cut] = mask
            rows.append(x)
        x = base.copy()
        x[np.arange(V) != 4321] = mask
        rows.append(x)
        rows.append(np.full(V, mask))
    mixed = np.full(V, -INF)
    mixed[[5, 77, 4999]] = low                                # a row of nothing but the two
    rows.append(mixed)
    for bad in (NAN, INF):
        for at in (0, 2500, V - 1):
            x = base.copy()
            x[at] = bad
            rows.append(x)
    some = base.copy()
    some[[3, 4]] = INF, -INF
    rows.append(some)
    nan = np.full(V, -INF)
    nan[9] = NAN
    rows.append(nan)
    rows.append(base.copy())
    n = len(rows)
    r = np.random.default_rng(1)
    logits = np.array(rows)
    for T in (None, [0.0] * n, [0.6] * n):
        run(dec, Verifying([1] * n, logits, [0] * n, [0.0] * n, r.random(n), T, dtype=dtype, pad=1))
        # each judges a draft that the next one is drawn from, and each is a draft model's
        both = np.repeat(logits, 2, axis=0)
        tokens = np.tile([0, 4321], n)
        u = r.random(2 * n) * 0.2
        run(dec, Verifying([2] * n, both, tokens, u, r.random(n), T, dtype=dtype))
        run(dec, Verifying([2] * n, both, tokens, u, r.random(n), T, logits[::-1].copy(), list(range(n)), dtype=dtype))
        other = rows_of(33, n, V, dtype)
        run(dec, Verifying([2] * n, np.repeat(other, 2, axis=0), tokens, u, r.random(n), T, logits, list(range(n)), dtype=dtype))


def test_drafts_that_are_no_tokens_and_rows_that_are_not_there(dec):
    V = 100
    logits = rows_of(2, 12, V, "fp32")
    tokens = [0, -1, 5, 0, V, 5, 0, 2 ** 31 - 1, 5, 0, 7, 5]
    u = [0.0] * 12
    draft = rows_of(3, 8, V, "fp32")
    run(dec, Verifying([3] * 4, logits, tokens, u, [0.2, 0.4, 0.6, 0.8], dtype="fp32"))
    for starts in ([0, 2, 4, 6], [-1, 7, 8, -2 ** 31], [2 ** 31 - 1, 6, 7, -5]):
        run(dec, Verifying([3] * 4, logits, tokens, u, [0.2, 0.4, 0.6, 0.8], draft=draft, draft_rows=starts, dtype="fp32"))
    run(dec, Verifying([3] * 4, logits, tokens, u, [0.2, 0.4, 0.6, 0.8], draft=draft[:0], draft_rows=[0] * 4, dtype="fp32"))


@pytest.mark.parametrize("scale", [1e-3, 30.0, 1e4, 1e30])
def test_sizes_of_logits_and_temperatures(dec, scale):
    """Logits far apart and close together; temperatures from almost none to beyond any use, negative and NaN (greedy)."""
    T = [1.0, 1e-2, 1e-6, 1e-30, 1e-38, 1e3, 1e9, 1e30, 1e35, INF, -1.0, NAN, 0.0]
    n, V = len(T), 900
    logits = rounded(scale * np.random.default_rng(int(scale) % 97).normal(0, 1, (n, V)), "fp32")
    logits[:, 10] = -INF
    x = Verifying([1] * n, logits, [0] * n, [0.0] * n, np.linspace(0.01, 0.99, n), T, dtype="fp32")
    dec.verify(x.c)
    torch.cuda.synchronize()
    # (a log-probability of (l - top) / T in the thousands is known to 2^-24 of its size, which check() allows for)
    x.exact = dec.exact
    x.check(scale)


def test_the_first_of_equal_logits(dec):
    """Greedy: among many equal ones, wherever they lie, the first."""
    V = 9000
    logits = rows_of(5, 6, V, "bf16", 1.0)
    for i, at in enumerate([(0, 8999), (7, 8), (2047, 2048), (8998, 8999), (4096, 5000, 6000), (1, 2, 3)]):
        logits[i, list(at)] = 50.0
    x = run(dec, Verifying([1] * 6, logits, [0] * 6, [0.0] * 6, [0.9] * 6, [0.0] * 6))
    assert x.next.tolist() == [0, 7, 2047, 8998, 4096, 1]


def test_bad_offsets(dec):
    """Sequences whose rows are not there count as having none."""
    logits = rows_of(5, 6, 40, "fp32")
    x = Verifying([2, 2, 2], logits, [1] * 6, [0.0] * 6, [0.5] * 3, dtype="fp32")
    x.cu.copy_(torch.tensor([0, 2, 9, 6], dtype=torch.int32))
    x.cu_host[:] = [0, 2, 9, 6]
    dec.verify(x.c)
    torch.cuda.synchronize()
    assert x.accepted.tolist()[1:] == [0, 0] and x.next.tolist()[1:] == [-1, -1]
    assert x.out.tolist()[2:] == [-77] * 4 and x.next.tolist()[0] >= 0


def test_nothing_to_verify(dec):
    e = torch.zeros((0, 50), device=DEV)
    i, f = (lambda *s: torch.full(s, -77, dtype=torch.int32, device=DEV)), (lambda *s: torch.zeros(s, device=DEV))
    accepted, nexts, cu = i(3), i(3), torch.zeros(4, dtype=torch.int32, device=DEV)
    dec.verify(ra.verify_from_tensors(e, cu, i(0), f(0), f(3), accepted, i(0), f(0), nexts))
    torch.cuda.synchronize()
    assert accepted.tolist() == [0] * 3 and nexts.tolist() == [-1] * 3
    dec.verify(ra.verify_from_tensors(f(2, 50), cu[:1], i(2), f(2), f(0), i(0), i(2)))


def test_only_what_is_asked_for_is_written(dec):
    x = drafting(6, [3, 2, 4], 333)
    x.c.out_logprobs = x.c.next_tokens = None
    dec.verify(x.c)
    torch.cuda.synchronize()
    assert (x.lps == 77).all() and (x.next == -77).all()
    x.lps.copy_(torch.tensor([l if l is not None else 77.0 for l in __import__("step_util").verify(*x.host)[2]]))
    x.next.copy_(torch.tensor(__import__("step_util").verify(*x.host)[3]))
    x.check()


def test_same_bytes_every_time_and_on_another_stream(dec):
    x = drafting(12, [5] * 40, 20011)
    dec.verify(x.c)
    torch.cuda.synchronize()
    was = [t.clone() for t in (x.accepted, x.out, x.next, x.lps)]
    for s in (None, torch.cuda.Stream(), None):
        for t in (x.accepted, x.out, x.next, x.lps):
            t.fill_(-5)
        torch.cuda.synchronize()
        dec.verify(x.c, stream=s)
        torch.cuda.synchronize()
        for a, b in zip(was, (x.accepted, x.out, x.next, x.lps)):
            assert torch.equal(a, b)


def test_refusals_enqueue_nothing(dec):
    x = drafting(3, [2, 3], 100)
    need = ra.rollout_attn_verify_workspace_size(dec.ctx, x.c)
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    for at, size, status in ((ws.data_ptr(), need - 1, ra.RA_ERR_WORKSPACE_TOO_SMALL), (ws.data_ptr() + 8, need, ra.RA_ERR_INVALID_ARG), (None, need, ra.RA_ERR_INVALID_ARG)):
        with pytest.raises(ra.RolloutAttnError) as e:
            ra.rollout_attn_verify(dec.ctx, x.c, at, size)
        assert e.value.status == status
    x.c.logits_dtype = 7
    with pytest.raises(ra.RolloutAttnError) as e:
        dec.verify(x.c)
    assert e.value.status == ra.RA_ERR_INVALID_ARG and "dtype" in str(e.value)
    torch.cuda.synchronize()
    assert (x.out == -77).all() and (x.accepted == -77).all()


@pytest.mark.parametrize("drafts,V,rows", [("logits", 4097, 5), ("guess", 4097, 4), ("guess", 12289, 1)])
def test_flat_rows(dec, drafts, V, rows):
    """Logits all but equal: every token is about as likely, thousands of borders lie close together, and no binary32 sum tells them
    apart."""
    n = 60
    x = drafting(V, [rows] * n, V, "fp32", drafts, near=0.01)
    x = Verifying(x.rows, rounded(0.01 * x.host[0], "fp32"), x.host[2], x.host[3], x.host[4], None, None if x.host[6] is None else rounded(0.01 * x.host[6], "fp32"),
                  x.host[7], dtype="fp32")
    run(dec, x)


def test_first_tokens_are_distributed_as_the_target_s(dec):
    """40 000 sequences of one draft each, all of the same two distributions: the first tokens' counts against the target's
    probabilities.  The sum of squares over what is expected has V - 1 = 11 degrees of freedom: above 40 in one of 27 000 tries, and the
    numbers are fixed."""
    n, V = 40000, 12
    r = np.random.default_rng(17)
    p_logits, q_logits = rounded(r.normal(0, 1, V), "fp32"), rounded(r.normal(0, 1, V), "fp32")
    p, q = distribution(p_logits, 1.0), distribution(q_logits, 1.0)
    drafts = r.choice(V, n, p=q)
    tokens = np.stack([np.zeros(n, dtype=np.int64), drafts], axis=1).reshape(-1)
    f = lambda x: torch.tensor(np.asarray(x, dtype=np.float32), device=DEV)
    i = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)
    logits, draft = f(p_logits).expand(2 * n, V).contiguous(), f(q_logits).expand(n, V).contiguous()
    out, accepted = i(np.zeros(2 * n)), i(np.zeros(n))
    dec.verify(ra.verify_from_tensors(logits, i(2 * np.arange(n + 1)), i(tokens), f(r.random(2 * n)), f(r.random(n)), accepted, out,
                                      draft_logits=draft, draft_rows=i(np.arange(n))))
    counts = np.bincount(out.cpu().numpy()[::2], minlength=V)
    assert ((counts - n * p) ** 2 / (n * p)).sum() < 40
    assert abs(float(accepted.float().mean()) - np.minimum(p, q).sum()) < 5 * 0.5 / n ** 0.5


@pytest.mark.parametrize("drafts", ["none", "guess"])
@pytest.mark.parametrize("V", [4097, 300001])
def test_open_draws_have_the_log_probability_of_binary64_sums(dec, V, drafts):
    """Numbers so near a border (1e-6; binary32 sums leave open what is within 9e-6 or more) that the row's sums are made again in binary64,
    at a temperature whose log2(e) / T is rounded by nearly half a step of binary32.  The log-probability is then rounded once, and off by
    2^-37 beside that, as if all sums had been binary64 from the start."""
    T = np.linspace(0.5, 2.0, 20001).astype(np.float32)
    c = 1.0 / np.log(2.0) / T.astype(np.float64)
    T = float(T[np.argmax(np.abs(c.astype(np.float32) / c - 1.0))])
    r = np.random.default_rng(V)
    small = np.log(0.4 / (V - 1)) * T
    row = rounded(np.concatenate([[0.0], small + 0.2 * T * r.normal(0, 1, V - 1)]), "fp32")
    p = distribution(row, float(np.float32(T)))
    x = 7                                                    # the guess that is turned down
    w = p.copy()
    if drafts == "guess":
        w[x] = 0.0
    border = np.cumsum(w)[0] / w.sum()
    at = [border - 1e-6, border - 3e-6, border + 1e-6]
    n, rows = len(at), 1 if drafts == "none" else 2
    v = Verifying([rows] * n, np.tile(row, (rows * n, 1)), [x] * (rows * n), [1.0] * (rows * n), at, [T] * n, dtype="fp32")
    dec.verify(v.c)
    v.exact = True
    v.check()
    assert v.next.tolist()[:2] == [0, 0] and v.next.tolist()[2] > 0
