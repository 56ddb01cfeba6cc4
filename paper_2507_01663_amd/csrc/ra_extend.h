// gfx950 kernels of the attention of chunks of new tokens over the paged cache.
//
// A sequence's n new tokens and the G query heads of a kv head are n * G rows that read the same keys: row r is token r / G,
// head r % G, and sees the keys up to L - n + r / G.  Packed that way 32 rows are a few tokens, so under the causal mask
// they need the same keys but for the last one or two stages of 32.
//
// A workgroup of four waves takes a block of up to 128 rows.  Many are bound by the matrix cores and the vector work between:
// 32 to a wave, all waves multiplying every stage of 32 keys that streams through one LDS ring:
//   S^T[key, row] = K . Q^T,   O^T[d, row] += V^T . P^T     (32x32x16 MFMA, binary32 sums, softmax running per row)
// Up to 64 are bound by the stream of pages: every wave multiplies stages of its own with all the rows, and what the waves have
// is added up in LDS (ex_narrow).  Kernels of its own do so where no sequence has more, and one has both ways where most
// sequences are far shorter than the longest.
//
// With q rows of D values, keys k_j and values v_j, a row's stages are taken with its running maximum m and sum l, all in
// binary32: s_j = scale <q, k_j> log2 e, p_j = 2^(s_j - m), l += sum p_j, o += sum p_j v_j; where a maximum exceeds m by more
// than 8, m moves there and o and l are multiplied by 2^(m_old - m_new) first.  p_j goes to the matrix cores as bf16, which
// rounds it (relative 2^-8 at most, the part of a result's error that its own rounding does not explain) and keeps l's unrounded sum;
// e4m3 codes go there as bf16 exactly, the page's scales into s_j and p_j before its rounding.
//
// What bounds it (stated sizes, MI355X): many rows, the vector instructions of the softmax beside the products and the clock
// that the card's power leaves: 2048 new tokens over 14 000, 64 heads on eight, 969 us, 1.04 PFLOP/s of the mask's products (e4m3
// 1167 us); 40 turns of 20 to 300 tokens over 1024 to 4000, 40 on eight, 431 us, 0.83 PFLOP/s (e4m3 505 us), an eighth of it items'
// starts and ends.  Few rows: 64 drafts of five tokens over up to 4000, 28 heads on four, 79.1 us, 4.1 TB/s (of four tokens, 28
// rows, 59.8 us; e4m3 60.1 and 43.4).  Batches of little work each: finding it (3 to 4 us), rows and first pages (3), parts'
// results (2) and their merge (7 to 10), beside the stages; about 16 us of some 50 to 60 are in none of these parts.
// Times here are of calls in a row whose inputs change; where two forms are compared both were timed in turn on one card.
//
// The work is a line of items, one per (sequence, kv head, block), each as long as it has stages, and the line is cut into
// as many spans of one length as workgroups are resident, so that ragged lengths load them alike.  Every workgroup finds its
// span by itself, from sums over the lengths.  An item that a cut goes through leaves its parts in the workspace, and a
// second kernel adds them up; items so short that cutting them would not pay are not cut: the cut moves to their nearer
// end.
#pragma once
#include "ra_chunk.h"
#include "ra_prefill.h"

namespace ra {

constexpr int kExWaves = 4;

// The kernels' arguments: what the search for a workgroup's work needs first is in registers when a wave starts, the rest is
// asked for at once.
#define EX_PARAMS                                                                                                               \
    const int32_t *__restrict__ cu, const int32_t *__restrict__ seq_lens, int B, int T, int max_chunk, int max_pages, int group, int Hkv, \
        uint32_t magic_g, int spans, ExtendLaunch given
#define EX_TAKE(a)                                                                                                             \
    ExtendLaunch a = given;                                                                                                     \
    a.cu = cu, a.seq_lens = seq_lens, a.B = B, a.T = T, a.max_chunk = max_chunk, a.max_pages = max_pages, a.G = group, a.Hkv = Hkv; \
    a.magic_g = magic_g, a.spans = spans;                                                                                       \
    touch_lines(given)
#define EX_GIVE(a) (a).cu, (a).seq_lens, (a).B, (a).T, (a).max_chunk, (a).max_pages, (a).G, (a).Hkv, (a).magic_g, (a).spans, (a)
constexpr int kExRows = kPfRows * kExWaves; // rows of a block

// ---- the line of items and its spans ------------------------------------------------------------------

struct ExSeq {
    int t0, n, L;  // first packed token, new tokens (up to max_chunk), tokens in all up to the last of them
    int blocks, cost, fixed; // blocks of a kv head; the length of each on the line (stages, the mean of the sequence's blocks, and ex_fixed)
};

// What an item costs beside its stages, in stages: finding it, its query rows, the first trip to memory, its results.  (8 to 9 us
// beside 0.7 to 1.0 for a stage that waves share, 5 beside 0.28 for one of few rows: 96 short turns, D = 64, e4m3, with 8 58.9 us, with
// 4 60.7.  A kernel that has both is the faster with 4 for either, 51.2 us against 55.6: the two kinds share compute units.)
constexpr int kExFixedMany = 8, kExFixedFew = 4;
__host__ __device__ __forceinline__ int ex_fixed(int most, bool two) { return most > 64 && !two ? kExFixedMany : kExFixedFew; }
constexpr int kExEdge = 2; // no part of an item is shorter than this (a span is longer than ex_fixed + 2 kExEdge)

__device__ __forceinline__ int ex_uni(int x) { return __builtin_amdgcn_readfirstlane(x); } // (a quotient comes from the vector unit)
// x / y for 0 <= x < 2^30, y > 0, both the wave's: the quotient by the reciprocal in binary32 is off by x / y 2^-22 at most, the
// remainder's by less than one, and a last comparison settles that.  (A quarter of the instructions of the compiler's.)
__device__ __forceinline__ int ex_div(int x, int y)
{
    const float inv = __builtin_amdgcn_rcpf((float)y);
    int q = (int)((float)x * inv);
    q += (int)((float)(x - q * y) * inv);
    const int r = x - q * y;
    return ex_uni(q + (r >= y) - (r < 0));
}

__device__ __forceinline__ int ex_div_g(const ExtendLaunch &a, int r) { return pf_div(r, a.G, a.magic_g); }

// Stages that block j of a sequence needs: up to the one with its last row's last key.
__device__ __forceinline__ int ex_stages(const ExtendLaunch &a, const ExSeq &s, int j)
{
    int last = ex_div_g(a, kExRows * (j + 1) - 1);
    last = s.L - s.n + (last < s.n - 1 ? last : s.n - 1);
    return (last + 32) >> 5; // (last >= -n: no key at all gives a number of zero or less)
}
// ... where x is often below 64 y: the multiples of y up to x are counted.
__device__ __forceinline__ int ex_div_short(int x, int y)
{
    if (x >= 64 * y) return ex_div(x, y);
    return __popcll(__ballot((int)(threadIdx.x & 63) * y <= x)) - 1;
}

// The length on the line of a number of stages, where sequences have up to so many rows: few rows take four at a time.
__host__ __device__ __forceinline__ int ex_weight(int stages, int most) { return most > 64 ? stages : stages * (most > 32 ? 14 : 9) >> 5; }

// Where most sequences are far shorter than the longest: does one of n tokens have few rows?
__device__ __forceinline__ bool ex_few(const ExtendLaunch &a, int n) { return a.two && n * a.G <= 32; }

// What the sequence of t0, t1 (where its chunk starts and ends) and length L is.  (A workgroup comes past everything up to its
// first keys once and alone, an instruction after the other: they are few.)
__device__ __forceinline__ ExSeq ex_sequence(const ExtendLaunch &a, int t0, int t1, int L)
{
    ExSeq s = {0, 0, 0, 0, 0, 0};
    const int n = t1 - t0, most = a.max_pages * kPage;
    if (t0 < 0 || t0 > a.T || n <= 0 || n > a.T - t0) return s;
    s.t0 = t0;
    s.n = n < a.max_chunk ? n : a.max_chunk;
    s.L = (L < 0 ? 0 : (L < most ? L : most)) - (n - s.n);
    s.L = s.L > 0 ? s.L : 0; // (none sees a key then)
    s.blocks = (s.n * a.G + kExRows - 1) / kExRows;
    const int mean = (s.L - (s.n >> 1) + 48) >> 5; // keys that a row sees, in stages
    const int most_rows = ex_few(a, s.n) ? 32 : a.max_chunk * a.G;
    s.fixed = ex_fixed(most_rows, a.two);
    s.cost = s.fixed + 1 + (mean > 0 ? ex_weight(mean, most_rows) : 0);
    return s;
}
__device__ __forceinline__ ExSeq ex_sequence(const ExtendLaunch &a, int b)
{
    return b < a.B ? ex_sequence(a, a.cu[b], a.cu[b + 1], a.seq_lens[b]) : ExSeq{0, 0, 0, 0, 0, 0};
}

// The line: lane c has chunk c of the sequences (64 of them, or a multiple of that in a very large batch).  Of a batch of up to
// 512, `known` keeps in LDS what the first search for a place needs; every wave writes all of it, the same values to the same
// place.
constexpr int kExKnown = 512;
struct ExKnown {
    int4 rec[kExKnown]; // {start on the line, -, first packed token, new tokens}
    int len[kExKnown];
    int2 rank[kExKnown]; // {class, blocks of the class before}
};
constexpr int kExClasses = 4; // items that are left whole begin with the longest, in so many classes of length
static_assert(sizeof(ExKnown) <= 3 * Geo<64, 2>::kStage, "it fits the smallest ring");

// Where some sequences have few rows and some have many (TWO), they are two lines, and the spans are divided between them.
template <bool TWO> struct ExLine {
    int lane, sub, chunks;   // sixty-fours of sequences in a chunk
    int unit;                // items are left whole (see measure)
    int few, base;           // which of two lines it is, and the number of its first span
    int before, total;       // start of this lane's chunk
    int before_few, total_few; // (the other line's, as long as both are measured)
    int blocks;              // blocks of one kv head, of all sequences
    int ranked[kExClasses], ranks[kExClasses]; // of an order by length: blocks of a class before this lane's chunk, and in all
    int q, r, spans, cut;    // span k starts at q k + min(k, r), before cuts are moved; items up to `cut` are not cut

    __device__ __forceinline__ void measure(const ExtendLaunch &a, ExKnown *known)
    {
        lane = threadIdx.x & 63;
        before = total = before_few = total_few = blocks = few = base = 0;
        int longest = 0;
        sub = 1;
        auto add = [&](const ExSeq &s) __attribute__((always_inline)) {
            int tc, tb;
            const int length = a.Hkv * s.blocks * s.cost;
            const bool other = TWO && ex_few(a, s.n);
            int at = total + wave_scan(other ? 0 : length, lane, tc);
            total += tc;
            if (TWO) {
                const int at_few = total_few + wave_scan(other ? length : 0, lane, tc);
                total_few += tc;
                at = other ? at_few : at;
            }
            (void)wave_scan(s.blocks, lane, tb);
            blocks += tb;
            longest = longest > s.cost ? longest : s.cost;
            return at;
        };
        if (a.B <= kExKnown) {
            chunks = (a.B + 63) >> 6;
            constexpr int AT = 2;
#pragma unroll 1
            for (int c0 = 0; c0 < chunks; c0 += AT) {
                int t0[AT], t1[AT], len[AT];
#pragma unroll
                for (int i = 0; i < AT; i++) {
                    const int b = 64 * (c0 + i) + lane;
                    t0[i] = t1[i] = len[i] = 0;
                    if (b < a.B) t0[i] = a.cu[b], t1[i] = a.cu[b + 1], len[i] = a.seq_lens[b];
                }
#pragma unroll
                for (int i = 0; i < AT; i++) {
                    if (c0 + i >= chunks) break;
                    const ExSeq s = ex_sequence(a, t0[i], t1[i], len[i]);
                    if (lane == c0 + i) before = total, before_few = total_few;
                    const int at = add(s);
                    known->rec[64 * (c0 + i) + lane] = make_int4(at, 0, s.t0, s.n);
                    known->len[64 * (c0 + i) + lane] = s.L;
                }
            }
        } else {
            sub = (a.B + 4095) >> 12;
            chunks = ex_div(a.B + 64 * sub - 1, 64 * sub);
#pragma unroll 1
            for (int c = 0; c < chunks * sub; c++) {
                if (lane * sub == c) before = total, before_few = total_few;
                (void)add(ex_sequence(a, 64 * c + lane));
            }
        }
        if (lane >= chunks) before = before_few = INT32_MAX;
        const int sum = total + total_few;
        spans = a.spans;
        if (sum < a.least * a.spans) {
            spans = ex_div(sum, a.least);
            spans = spans < 1 ? 1 : spans;
        }
        divide(a, sum);
        // Many items, none of them longer than what a workgroup has on average: they are left whole, a workgroup for each.  (40
        // turns, 2288 items: 431 us, cut into spans 528; 64 over 100 to 2000, 32 heads on eight, D = 64, 200 and 237.)
        unit = a.B <= kExKnown && blocks * a.Hkv >= 2 * a.spans && !__any(longest > q);
        if (!unit) return;
        // (what is started last should be short: by length, in classes of a quarter of the longest; the 40 turns 441 -> 431 us)
#pragma unroll
        for (int sh = 32; sh >= 1; sh >>= 1) {
            const int o = __shfl_xor(longest, sh);
            longest = longest > o ? longest : o;
        }
#pragma unroll
        for (int k = 0; k < kExClasses; k++) ranked[k] = INT32_MAX, ranks[k] = 0;
#pragma unroll 1
        for (int c = 0; c < chunks; c++) {
            const int b = 64 * c + lane;
            const int4 rec = known->rec[b];
            const ExSeq s = ex_sequence(a, rec.z, rec.z + rec.w, known->len[b]);
            const int cls = 4 * s.cost >= 3 * longest ? 0 : 2 * s.cost >= longest ? 1 : 4 * s.cost >= longest ? 2 : 3;
            int mine = 0;
#pragma unroll
            for (int k = 0; k < kExClasses; k++) {
                int t;
                const int at = ranks[k] + wave_scan(cls == k ? s.blocks : 0, lane, t);
                if (cls == k) mine = at;
                if (lane == c) ranked[k] = ranks[k];
                ranks[k] += t;
            }
            known->rank[b] = make_int2(cls, mine);
        }
    }
    __device__ __forceinline__ void divide(const ExtendLaunch &a, int length)
    {
        q = ex_div(length, spans);
        r = length - q * spans;
        cut = q >> 3 > a.least ? q >> 3 : a.least;
    }
    // The span of the workgroup that is number `at` of a die, counted from the line's first (-1: there is none).  `number`: of
    // all spans, and for workgroups without one the numbers that are left.
    __device__ __forceinline__ int take(const ExtendLaunch &a, int die, int at, int &number)
    {
        int of_few = 0; // spans of the line of few rows, and after that of the other; both a multiple of eight, or up to eight
        if (TWO && total_few > 0) {
            if (total == 0) {
                of_few = spans;
            } else {
                const int n = ex_uni((int)((float)spans * ((float)total_few / (float)(total + total_few)) + 0.5f));
                const int most_few = ex_div(total_few, a.least), most = ex_div(total, a.least);
                if (spans < 16) {
                    of_few = n < 1 ? 1 : n < 8 ? n : 8;
                    spans = spans - of_few < 1 ? 1 : spans - of_few < 8 ? spans - of_few : 8;
                } else {
                    spans &= ~7;
                    of_few = (n + 4) & ~7;
                    of_few = of_few < 8 ? 8 : of_few < spans - 8 ? of_few : spans - 8;
                    spans -= of_few;
                }
                of_few = of_few < most_few ? of_few : most_few > 1 ? most_few : 1;
                spans = spans < most ? spans : most > 1 ? most : 1;
            }
            const int per = (of_few + 7) >> 3;
            if (at < per || total == 0) few = 1, total = total_few, before = before_few, spans = of_few;
            else at -= per, base = 8 * per;
            divide(a, total);
        }
        const int per = (spans + 7) >> 3, k = die * per + at;
        if (at < per) number = base + k;
        return at < per && k < spans && total > 0 ? k : -1;
    }
    __device__ __forceinline__ int raw(int k) const { return q * k + (k < r ? k : r); }
    // The last span that starts at y or before it, but for cuts that move.
    __device__ __forceinline__ int span_of(int y) const
    {
        const int big = r * (q + 1);
        const bool in_big = y < big;
        return (in_big ? 0 : r) + ex_div(in_big ? y : y - big, in_big ? q + 1 : q);
    }
    // The first and the last span that an item which is cut and lies from x0 to x1 has a part in (cuts near its ends move there).
    __device__ __forceinline__ int first_of(int x0, const ExSeq &s) const { return span_of(x0 + s.fixed + kExEdge - 1); }
    __device__ __forceinline__ int last_of(int x1) const
    {
        const int k = span_of(x1 - 1);
        return x1 - raw(k) < kExEdge ? k - 1 : k;
    }
    // Where a cut at x goes in the item of that length that starts at x0: nowhere into short items, and not so near an end of
    // others that a part would be next to nothing.
    __device__ __forceinline__ int moved(int x, int x0, const ExSeq &s) const
    {
        const int y = x - x0, cost = s.cost, left = cost - y;
        const bool down = cost > cut ? y < s.fixed + kExEdge : y < left, up = cost > cut ? left < kExEdge : true;
        return down ? x0 : up ? x0 + cost : x;
    }
};

// A place on the line: an item of a sequence.
struct ExPlace {
    int b, item, x0; // the sequence, its item (kv head * blocks + number), the item's start
    ExSeq s;         // (cost: the item's length on the line)
};

__device__ __forceinline__ void ex_place(const ExtendLaunch &a, const ExSeq &s, int base, int l, ExPlace &p)
{
    p.b = base + l;
    const int t0 = __builtin_amdgcn_readlane(s.t0, l);
    p.s = ex_sequence(a, t0, t0 + __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.L, l));
}

// The item that x lies in (0 <= x < total).
template <bool TWO>
__device__ __forceinline__ void ex_find(const ExtendLaunch &a, const ExLine<TWO> &line, const ExKnown *known, int x, ExPlace &p)
{
    const int c = 63 - __builtin_clzll(__ballot(line.before <= x));
    int base = 64 * c, before;
    ExSeq s = {0, 0, 0, 0, 0, 0};
    if (known) {
        const int4 rec = known->rec[base + line.lane];
        s.t0 = rec.z, s.n = rec.w, s.L = known->len[base + line.lane], before = rec.x;
    } else {
        int start = __builtin_amdgcn_readlane(line.before, c);
#pragma unroll 1
        for (int i = 0;; i++) {
            base = (c * line.sub + i) * 64;
            s = ex_sequence(a, base + line.lane);
            if (TWO && ex_few(a, s.n) != (line.few != 0)) s.n = s.blocks = 0;
            int t;
            before = start + wave_scan(a.Hkv * s.blocks * s.cost, line.lane, t);
            if (x < start + t || i + 1 == line.sub) break;
            start += t;
        }
    }
    const int l = 63 - __builtin_clzll(__ballot(s.n > 0 && before <= x && (!TWO || ex_few(a, s.n) == (line.few != 0))));
    ex_place(a, s, base, l, p);
    const int y = x - __builtin_amdgcn_readlane(before, l);
    p.item = ex_div_short(y, p.s.cost);
    p.x0 = x - y + p.item * p.s.cost;
}

// The sequence that block x of one kv head lies in, in the order by length; returns x's distance from its start.
template <bool TWO>
__device__ __forceinline__ int ex_find_ranked(const ExtendLaunch &a, const ExLine<TWO> &line, const ExKnown *known, int x, ExPlace &p)
{
    int cls = 0, ranked = line.ranked[0];
#pragma unroll
    for (int k = 0; k + 1 < kExClasses; k++) {
        if (cls == k && x >= line.ranks[k]) x -= line.ranks[k], cls = k + 1, ranked = line.ranked[k + 1];
    }
    const int c = 63 - __builtin_clzll(__ballot(ranked <= x)), b = 64 * c + line.lane;
    const int4 rec = known->rec[b];
    const int2 rank = known->rank[b];
    const ExSeq s = {rec.z, rec.w, known->len[b], 0, 0, 0};
    const int l = 63 - __builtin_clzll(__ballot(s.n > 0 && rank.x == cls && rank.y <= x));
    ex_place(a, s, 64 * c, l, p);
    return x - __builtin_amdgcn_readlane(rank.y, l);
}

// A part of an item that a workgroup works on.
struct ExPart {
    int kvh, row0, rows; // rows of the sequence and kv head in all
    int lo, hi;          // stages
    int slot;            // -1: the item is whole; else where its part goes
};

// The blocks of a (sequence, kv head) come from both ends in turn: their mean cost is the line's.
__device__ __forceinline__ ExPart ex_part(const ExtendLaunch &a, const ExPlace &p, int y0, int y1, int span)
{
    ExPart t;
    t.kvh = ex_div_short(p.item, p.s.blocks);
    const int jj = p.item - t.kvh * p.s.blocks, j = jj & 1 ? p.s.blocks - 1 - (jj >> 1) : jj >> 1;
    t.row0 = kExRows * j;
    t.rows = p.s.n * a.G;
    int stages = ex_uni(ex_stages(a, p.s, j));
    stages = stages < 0 ? 0 : stages;
    // (a place inside the item, in proportion: the same for the two parts that it divides)
    auto stage_at = [&](int y) __attribute__((always_inline)) {
        return ex_uni((int)((float)stages * ((float)(y - p.s.fixed) * __builtin_amdgcn_rcpf((float)(p.s.cost - p.s.fixed)))));
    };
    t.lo = y0 == 0 ? 0 : stage_at(y0);
    t.hi = y1 == p.s.cost ? stages : stage_at(y1);
    t.slot = y0 == 0 ? (y1 == p.s.cost ? -1 : 2 * span + 1) : 2 * span;
    return t;
}

// Goes through the parts that the workgroup works on; `work` is called with each.  Workgroups are dealt to the eight dies
// round-robin, each with an L2 of its own.
// Items that are left whole: with gg = gcd(Hkv, 8), a die takes the kv heads congruent to it mod gg, and the 8 / gg dies that
// take the same heads take their items in turn, so that every die has its share of every sequence, and blocks that read the
// same keys run side by side on few of them.
// Else: a die takes neighbouring spans.  Also tells the merge which spans begin inside an item: desc[2 k], desc[2 k + 1] =
// {first packed token, first row, rows, kv head}, {first span of the item or -1, its last, -, -}.
// `work_few`: the same for sequences of few rows, where there are both (TWO).
template <bool TWO, typename F, typename FewF> __device__ __forceinline__ void ex_walk(const ExtendLaunch &a, uint8_t *lds, F &&work, FewF &&work_few)
{
    const int die = (int)blockIdx.x & 7, at = (int)blockIdx.x >> 3;
    const int gg_shift = (a.Hkv & 7) == 0 ? 3 : (a.Hkv & 3) == 0 ? 2 : (a.Hkv & 1) == 0 ? 1 : 0, s_shift = 3 - gg_shift, heads = a.Hkv >> gg_shift;
    const int first_head = die & ((1 << gg_shift) - 1), share = (at << s_shift) + (die >> gg_shift);
    const ExKnown *known = a.B <= kExKnown ? (ExKnown *)lds : nullptr;
    ExLine<TWO> line;
    ExPlace p;
    ExPart part;
    p.item = 0, p.x0 = 0;
    int x = 0, end = 0, k = -1, number = blockIdx.x;
    int2 ends = {-1, 0};
    bool whole = false; // one item, and nothing else
    int4 begun = {0, 0, 0, 0};
    if (a.direct) {
        // Every item is short: a workgroup for each, and no line.  Blocks are numbered without counting them: sequence b's
        // are given the numbers from cu[b] G / kExRows + b on, which leaves it as many as it can have.
        const int block = ex_div_short(share, heads), lane = threadIdx.x & 63;
        int j = 0;
        p.b = block;
        if (!a.few) {
            p.b = -1;
#pragma unroll 1
            for (int base = 0; base < a.B; base += 64) {
                const int start = base + lane < a.B ? (int)((int64_t)a.cu[base + lane] * a.G / kExRows) + base + lane : INT32_MAX;
                const unsigned long long m = __ballot(start <= block);
                if (!m) break;
                const int l = 63 - __builtin_clzll(m);
                p.b = base + l, j = block - __builtin_amdgcn_readlane(start, l);
                if (l < 63) break;
            }
        }
        if (p.b < 0 || p.b >= a.B) return;
        p.s = ex_sequence(a, uniform_load(a.cu, p.b), uniform_load(a.cu, p.b + 1), uniform_load(a.seq_lens, p.b));
        if (j < 0 || j >= p.s.blocks) return;
        part.kvh = ((share - block * heads) << gg_shift) + first_head;
        part.row0 = kExRows * j, part.rows = p.s.n * a.G;
        part.lo = 0, part.hi = ex_stages(a, p.s, j), part.slot = -1;
        part.hi = part.hi < 0 ? 0 : part.hi;
        whole = true, end = 1;
    } else {
        line.measure(a, (ExKnown *)lds);
        if (!line.unit) k = line.take(a, die, at, number);
        if (line.unit) {
            // (a workgroup for each item: there are as many, if the call's sizes are what they say)
            const int block = ex_div_short(share, heads);
            if (block < line.blocks) {
                const int i = share - (block - ex_find_ranked(a, line, known, block, p)) * heads; // the sequence's items: its blocks times heads
                const int h = ex_div_short(i, p.s.blocks);
                p.item = i + ((h << gg_shift) + first_head - h) * p.s.blocks;
                part = ex_part(a, p, 0, p.s.cost, 0);
                whole = true, end = 1;
            }
        } else if (k >= 0) {
            // `end` is moved where the span gets to it
            end = k + 1 < line.spans ? line.raw(k + 1) : line.total, x = line.raw(k);
            ex_find(a, line, known, x, p);
            x = line.moved(x, p.x0, p.s);
            if (x == p.x0 + p.s.cost) {
                if (p.item + 1 < a.Hkv * p.s.blocks) p.item++, p.x0 = x;
                else if (x < end) ex_find(a, line, known, x, p);
            }
        }
    }
    auto go = [&](auto &&work) __attribute__((always_inline)) {
        bool first = !a.direct;
        while (x < end) {
            int next = end;
            if (!whole) {
                const int x1 = p.x0 + p.s.cost;
                if (end < x1) end = line.moved(end, p.x0, p.s);
                if (x >= end) break;
                next = x1 < end ? x1 : end;
                part = ex_part(a, p, x - p.x0, next - p.x0, number);
                if (x > p.x0) {
                    begun = make_int4(p.s.t0, part.row0, part.rows, part.kvh);
                    ends = make_int2(line.base + line.first_of(p.x0, p.s), line.base + line.last_of(x1));
                }
            }
            if (first) __syncthreads(); // (what the waves know of the line makes room for the ring)
            first = false;
            work(p, part);
            x = next;
            if (x >= end) break;
            if (p.item + 1 < a.Hkv * p.s.blocks) p.item++, p.x0 = x;
            else ex_find(a, line, nullptr, x, p);
        }
    };
    if (TWO && (whole ? ex_few(a, p.s.n) : line.few != 0)) go(work_few);
    else go(work);
    if (!a.direct && threadIdx.x == 0 && number < a.spans) { // (every span is answered for, also one that does not exist)
        a.desc[2 * number] = begun;
        a.desc[2 * number + 1] = make_int4(ends.x, ends.y, 0, 0);
    }
}

// ---- values that a row does not see ---------------------------------------------------------------------
//
// In the stages that the causal mask cuts, a row's weight of a later token is zero, and zero times an infinite or NaN value
// is NaN.  Where a V operand of such a stage holds one (which is looked for there alone), the product is made without these
// values, and what they do to the rows that see them is added apart: a product of "infinite, or NaN" with "seen" for either
// sign, and an infinity for every place where it is not zero.  NaN has both.
//
// The scale of an e4m3 page may be infinite or NaN as well (an appended infinity makes it infinite).  Where one of such a stage is
// (which is looked for there alone), the page's scores are multiplied by it before the mask, so that later tokens' are -inf, and
// V's scale has no part in the weights, all zero, of a row that does not see the page.  (A row that sees any of it is not finite
// anyway: finite values have code zero there.  By the weights one by one instead: 64 drafts of five, e4m3, 59 -> 67 us; so 60.)

__device__ __forceinline__ bool ex_odd(bf16x8 v)
{
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; i++) odd = odd || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
// Is one of a stage's scales infinite or NaN?  (None is negative.)
__device__ __forceinline__ bool ex_odd(float k0, float k1, float v0, float v1) { return __any(!(k0 + k1 + v0 + v1 < INFINITY)); }
// Takes K scales that are into the stage's scores: of the page's keys that the lane's row sees; the others' are -inf.
__device__ __forceinline__ void ex_scale_seen(f32x16 &s, float k0, float k1, int key, int lim, int hh)
{
#pragma unroll
    for (int e = 0; e < 16; e++) {
        const float k = e < 8 ? k0 : k1;
        if (!(k < INFINITY)) s[e] = key + 8 * (e >> 2) + 4 * hh + (e & 3) > lim ? -INFINITY : s[e] * k;
    }
}
// v without them; plus, minus: one where v has an infinity of that sign or a NaN.
__device__ __forceinline__ bf16x8 ex_even(bf16x8 v, u32x4 &plus, u32x4 &minus)
{
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        unsigned keep = 0, up = 0, down = 0;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const unsigned x = (w[i] >> (16 * h)) & 0xffffu, m = x & 0x7fffu;
            if (m < 0x7f80u) keep |= x << (16 * h);
            if (x == 0x7f80u || m > 0x7f80u) up |= 0x3f80u << (16 * h);
            if (x == 0xff80u || m > 0x7f80u) down |= 0x3f80u << (16 * h);
        }
        w[i] = keep, plus[i] = up, minus[i] = down;
    }
    return __builtin_bit_cast(bf16x8, w);
}
// The second operand of such a product: one where the lane's row sees the key.  Slot e of half hh of the sixteen keys from
// `key` on is key 8 (e / 4) + 4 hh + e % 4.
__device__ __forceinline__ bf16x8 ex_seen(int key, int lim, int hh)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        w[i] = 0;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int e = 2 * i + h;
            if (key + 8 * (e >> 2) + 4 * hh + (e & 3) <= lim) w[i] |= 0x3f80u << (16 * h);
        }
    }
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ void ex_add_odd(f32x16 &o, u32x4 of, bf16x8 seen, float infinity)
{
    f32x16 w;
#pragma unroll
    for (int e = 0; e < 16; e++) w[e] = 0.f;
    w = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, of), seen, w, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 16; e++) o[e] += w[e] > 0.f ? infinity : 0.f;
}

// ---- many rows ------------------------------------------------------------------------------------------

// Scale of a stage's first and second page for the scores (softmax scale and binary logarithm included), and for V.
struct ExScale {
    float k0, k1, v0, v1;
};

// One step of a wave's software pipeline: the weights of a stage (whose scores are st.s) and the scores of the next
// (NEXT; MASK: the causal mask cuts one of the two), then O += P V of the first and the maxima of the new scores.
// key, key_next: first keys of the two stages; lim: the last key that the lane's row sees.
// As pf_step, but for the scales of e4m3 pages (their codes lie in the ring as bf16, exactly) and what MASK does with V and with them.
template <int D, bool FP8, bool MASK, bool NEXT>
__device__ __forceinline__ void ex_step(PfState<D> &st, uint32_t k_next, uint32_t v_addr, const PfLane<D> &pl, const ExScale &sc, const ExScale &sn_,
                                        int key, int key_next, int lim)
{
    using G = Geo<D, 2>;
    typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
    typedef bf16x8 __attribute__((address_space(3))) * lds_bf16x8;
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const int hh = (threadIdx.x & 63) >> 5;
    constexpr int KS = D / 16, DT = D / 32;
#define EX_FENCE() __builtin_amdgcn_sched_barrier(0)
    EX_FENCE();
    constexpr int KA = KS < 4 ? KS : 4; // K operands are read four products ahead of their use
    bf16x8 kf[KS];
    uint32_t ka = k_next + (uint32_t)pl.k_base;
    asm volatile("" : "+v"(ka));
    if (NEXT) {
#pragma unroll
        for (int i = 0; i < KA; i++) kf[i] = *(lds_bf16x8)(ka ^ (uint32_t)(32 * i));
    }
    uint32_t vb = v_addr + (uint32_t)pl.v_base;
    asm volatile("" : "+v"(vb));
    s16x4 vr[DT][2][2];
    auto v_read = [&](int dt, int kk) {
#pragma unroll
        for (int rd = 0; rd < 2; rd++)
            vr[dt][kk][rd] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb ^ (uint32_t)pf_v_xor<D>(dt, rd)) + kk * G::kTile / 8);
    };
    EX_FENCE();
    const bool odd_scale = FP8 && (MASK || !NEXT) && ex_odd(sc.k0, sc.k1, sc.v0, sc.v1);
    float k0 = sc.k0, k1 = sc.k1, v0 = sc.v0, v1 = sc.v1;
    if (__builtin_expect(odd_scale, 0)) {
        ex_scale_seen(st.s, k0, k1, key, lim, hh);
        k0 = k0 < INFINITY ? k0 : 1.f, k1 = k1 < INFINITY ? k1 : 1.f;
        v0 = key > lim ? 1.f : v0, v1 = key + kPage > lim ? 1.f : v1;
    }
    u32x4 pw[2];
    float pprev = 0.f, acc0 = 0.f, acc1 = 0.f;
    auto w_item = [&](int k) {
        if (k < 16) {
            float pk = __builtin_amdgcn_exp2f(__builtin_fmaf(st.s[k], k < 8 ? k0 : k1, -st.m));
            if (k & 1) acc1 = k == 1 ? pk : acc1 + pk;
            else acc0 = k == 0 ? pk : acc0 + pk;
            if (FP8) pk *= k < 8 ? v0 : v1;
            if (k & 1) pw[k >> 3][(k >> 1) & 3] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{pprev, pk}), bf16x2));
            else pprev = pk;
        } else {
            st.lsum += acc0 + acc1;
        }
    };
    constexpr int NW = 17;
    f32x16 sn;
    // (Of two waves on a SIMD the one further on goes first, which keeps one in products while the other has its weights to make:
    // 2048 tokens over 14 000 1006 -> 968 us, 40 turns 443 -> 431, 96 short ones, e4m3, 60.5 -> 58.9; for the second half alone
    // 963, 433, 60.2, the same for all of a step 1002, 443, 59.5.)
    __builtin_amdgcn_s_setprio(1);
    if (NEXT) {
#pragma unroll
        for (int k = 0; k < 3; k++) w_item(k);
        EX_FENCE();
#pragma unroll
        for (int i = 0; i < KS; i++) {
            if (i == 0) {
#pragma unroll
                for (int e = 0; e < 16; e++) sn[e] = 0.f;
            }
            sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], st.qf[i], sn, 0, 0, 0);
            if (i + KA < KS) kf[i + KA] = *(lds_bf16x8)(ka ^ (uint32_t)(32 * (i + KA)));
#pragma unroll
            for (int w = 3 + i * (NW - 3) / KS; w < 3 + (i + 1) * (NW - 3) / KS; w++) w_item(w);
            if (i >= KS - DT) v_read((i - (KS - DT)) / 2, (i - (KS - DT)) % 2);
            EX_FENCE();
        }
    } else {
#pragma unroll
        for (int n = 0; n < DT; n++) v_read(n / 2, n % 2);
#pragma unroll
        for (int w = 0; w < NW; w++) w_item(w);
        EX_FENCE();
    }
    // item k: 0..3 the causal mask, 4..11 partial maxima, 12 the exchange, 13 the end
    float mx = 0.f, mx0 = 0.f, mn = 0.f;
    bool grew = false;
    auto m_item = [&](int k) {
        if (k < 4) {
            if (MASK) {
                const int kk = key_next + 8 * k + 4 * hh; // element e = 4 k + x is key 8 k + 4 hh + x of the stage
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    if (kk + x > lim) sn[4 * k + x] = -INFINITY;
                }
            }
        } else if (k == 4) {
            mx = max3(first_max(sn[0], sn[1]), sn[2], sn[2]);
        } else if (k < 8) {
            mx = max3(mx, sn[2 * k - 7], sn[2 * k - 6]); // k = 5..7: elements 3..8
        } else if (k < 11) {
            mx = max3(mx, sn[2 * k - 7], sn[2 * k - 6]); // k = 8..10: elements 9..14
        } else if (k == 11) {
            mx = max3(mx, sn[15], sn[15]);
        } else if (k == 12) {
            const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[1]));
        } else {
            mn = FP8 ? mx : mx * sn_.k0;
            grew = mn > st.m + kPfSlack;
            st.s = sn;
        }
    };
    // (two pages of unlike scales: their maxima apart, each scaled, then the larger)
    auto m_item8 = [&](int k) {
        if (k < 4) m_item(k);
        else if (k == 4) mx0 = max3(first_max(sn[0], sn[1]), sn[2], sn[3]);
        else if (k == 5) mx0 = max3(mx0, sn[4], sn[5]);
        else if (k == 6) mx0 = max3(mx0, sn[6], sn[7]);
        else if (k == 7) mx = max3(first_max(sn[8], sn[9]), sn[10], sn[11]);
        else if (k == 8) mx = max3(mx, sn[12], sn[13]);
        else if (k == 9) mx = max3(mx, sn[14], sn[15]);
        else if (k == 10) mx = fmaxf(mx0 * sn_.k0, mx * sn_.k1); // (-inf by a scale that is NaN: no part in the maximum)
        else if (k >= 12) m_item(k);
    };
    constexpr int NMI = NEXT ? 14 : 0, NPV = 2 * DT;
    __builtin_amdgcn_s_setprio(2);
#pragma unroll
    for (int n = 0; n < NPV; n++) {
        const int dt = n / 2, kk = n % 2;
        if (n + DT < NPV) v_read((n + DT) / 2, (n + DT) % 2);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(vr[dt][kk][0], vr[dt][kk][1], 0, 1, 2, 3, 4, 5, 6, 7));
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw[kk]);
        if ((MASK || !NEXT) && __builtin_expect(__any(ex_odd(vf)), 0)) {
            u32x4 plus, minus;
            const bf16x8 even = ex_even(vf, plus, minus), seen = ex_seen(key + 16 * kk, lim, hh);
            st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(even, pf, st.o[dt], 0, 0, 0);
            ex_add_odd(st.o[dt], plus, seen, INFINITY), ex_add_odd(st.o[dt], minus, seen, -INFINITY);
        } else {
            st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, st.o[dt], 0, 0, 0);
        }
#pragma unroll
        for (int w = n * NMI / NPV; w < (n + 1) * NMI / NPV; w++) {
            if (FP8) m_item8(w);
            else m_item(w);
        }
        EX_FENCE();
    }
    __builtin_amdgcn_s_setprio(0);
    if (NEXT) {
        if (__any(grew)) {
            mn = grew ? mn : st.m; // (row by row: a row's result is the same whatever the wave's other rows hold)
            const float alpha = __builtin_amdgcn_exp2f(st.m - mn);
            st.m = mn;
            st.lsum *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; dt++) st.o[dt] *= alpha;
        }
    }
#undef EX_FENCE
}

// ---- few rows -------------------------------------------------------------------------------------------
//
// A block of up to 32 NG rows keeps one or two waves busy with a stage that all four wait for.  Here every wave multiplies
// stages of its own (every fourth one of the part) with all the rows, as they land in a place of its own: K and V in turn,
// each asked for as soon as the operands before it are in registers, so that a wave has 32 keys on the way while it works on
// others and no wave waits for another.  What the waves have is added up in LDS.  The query rows, which all waves read, lie in
// LDS like a K tile.

template <int D, bool FP8> struct ExNarrowLds {
    using G = Geo<D, FP8 ? 1 : 2>;
    static constexpr int kWave = 4 * G::kTile;             // K and V of a stage, as stored
    static constexpr int kScales = kExWaves * kWave;        // e4m3: each wave's scales
    static constexpr int kNeeds = kScales + (FP8 ? kExWaves * 256 : 0);
    static constexpr int kRows = 2 * 32 * D * 2;            // the query rows, behind the ring in the waves' areas
    // in the end, over all of it: the waves' sums of 32 rows, 64 d of them at a time, and maximum and sum of these rows
    static constexpr int kSum = 32 * 64 * 4, kStats = kExWaves * kSum, kEnds = kStats + kExWaves * 32 * 8;
};

template <int D, bool FP8, int NG, typename LC>
__device__ __forceinline__ void ex_narrow(const ExtendLaunch &a, const ExPlace &p, const ExPart &t, const LC &lc, const PfLane<D> &pl, uint8_t *lds,
                                          uint8_t *areas, int lane, int wave)
{
    using G = Geo<D, 2>;
    using P = Geo<D, FP8 ? 1 : 2>;
    using X = ExNarrowLds<D, FP8>;
    typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
    typedef bf16x8 __attribute__((address_space(3))) * lds_bf16x8;
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef int __attribute__((ext_vector_type(2))) i32x2;
    typedef i32x2 __attribute__((address_space(3))) * lds_i32x2;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    constexpr int KS = D / 16, DT = D / 32, UM = G::kUnits - 1, PUM = P::kUnits - 1;
    const int n = lane & 31, hh = lane >> 5, shift = p.s.L - p.s.n;
    const uint32_t lds_addr = (uint32_t)(uintptr_t)lds, q_addr = (uint32_t)(uintptr_t)areas;
    const uint32_t k_addr = lds_addr + wave * X::kWave, v_addr = k_addr + 2 * P::kTile, scale_addr = lds_addr + X::kScales + 256 * wave;

    // the wave's stages of the part: wave, wave + 4, ...
    const int left = t.hi - t.lo - wave, mine = left > 0 ? (left + kExWaves - 1) / kExWaves : 0;
    const int32_t *const pages = a.table + (int64_t)p.b * a.max_pages;
    const int count = (p.s.L + kPage - 1) / kPage, last_page = count > 0 ? count - 1 : 0;
    const int64_t head_b = (int64_t)t.kvh * a.stride_head_b;
    auto page_id = [&](int i, int h) __attribute__((always_inline)) { // (a page that does not exist takes the last one's place, and none of its rows are read)
        const int g = 2 * (t.lo + wave + kExWaves * i) + h;
        return uniform_load(pages, g < last_page ? g : last_page);
    };
    int id0 = 0, id1 = 0, next0 = 0, next1 = 0; // pages of the stage whose K was asked for last, and of the one after it
    auto load_k = [&](int i) __attribute__((always_inline)) {
        const int nv = p.s.L - 32 * (t.lo + wave + kExWaves * i);
        id0 = next0, id1 = next1;
        if (i + 1 < mine) next0 = page_id(i + 1, 0), next1 = page_id(i + 1, 1);
        issue_tile<D, FP8 ? 1 : 2, true>(lc, a.k_pool + (int64_t)id0 * a.stride_page_b + head_b, nv, k_addr, a.zeros);
        issue_tile<D, FP8 ? 1 : 2, true>(lc, a.k_pool + (int64_t)id1 * a.stride_page_b + head_b, nv - kPage, k_addr + P::kTile, a.zeros);
        if (FP8) { // lanes 0..3 bring K and V scale of the first page, K and V scale of the second
            const void *src = a.zeros;
            if (lane < 4 && ((lane & 2) ? nv - kPage : nv) > 0) src = ((lane & 1) ? a.v_scale : a.k_scale) + (int64_t)((lane & 2) ? id1 : id0) * a.Hkv + t.kvh;
            dma4(src, scale_addr);
        }
    };
    auto load_v = [&](int i) __attribute__((always_inline)) { // (before K of the stage after it)
        const int nv = p.s.L - 32 * (t.lo + wave + kExWaves * i);
        issue_tile<D, FP8 ? 1 : 2, true>(lc, a.v_pool + (int64_t)id0 * a.stride_page_b + head_b, nv, v_addr, a.zeros);
        issue_tile<D, FP8 ? 1 : 2, true>(lc, a.v_pool + (int64_t)id1 * a.stride_page_b + head_b, nv - kPage, v_addr + P::kTile, a.zeros);
    };
    constexpr int NK = 2 * P::kDmaPerTile + (FP8 ? 1 : 0), NV = 2 * P::kDmaPerTile; // loads of a stage's K and of its V
    if (mine > 0) next0 = page_id(0, 0), next1 = page_id(0, 1);
    __syncthreads(); // (the ring and the areas of the part before have been read)
    if (mine > 0) load_k(0), load_v(0);
    {
        constexpr int UNITS = 32 * NG * G::kUnits;
#pragma unroll
        for (int x = 0; x < UNITS / (64 * kExWaves); x++) {
            const int u = 64 * kExWaves * x + (int)threadIdx.x, r = u / G::kUnits, c = u % G::kUnits;
            int row = t.row0 + r;
            row = row < t.rows ? row : t.rows - 1;
            const int token = ex_div_g(a, row);
            const uint4 w = *(const uint4 *)(a.q + (int64_t)(p.s.t0 + token) * a.q_stride + (t.kvh * a.G + row - token * a.G) * D + 8 * c);
            *(uint4 *)(areas + (r >> 4) * G::kTile + 16 * ((r & 15) * G::kUnits + (c ^ (swz(r & 15) & UM)))) = w;
        }
    }
    __syncthreads();

    int lim[NG];
    f32x16 o[NG][DT];
    float m[NG], l[NG];
#pragma unroll
    for (int g = 0; g < NG; g++) {
        const int row = t.row0 + 32 * g + n;
        lim[g] = shift + ex_div_g(a, row < t.rows ? row : t.rows - 1);
        m[g] = kPfLowest, l[g] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) {
#pragma unroll
            for (int e = 0; e < 16; e++) o[g][dt][e] = 0.f;
        }
    }
    const int first_lim = shift + ex_div_g(a, t.row0); // (the first row sees the least)
    // e4m3: sixteen codes of a K row at a time are the operands of two k-steps, d = 32 i + 16 hh .. + 7 and + 8 .. + 15; so are Q's
    const int r16 = n & 15;
    const int kq_base = FP8 ? (n >> 4) * G::kTile + G::kRowBytes * r16 + 16 * ((swz(r16) & UM) ^ (2 * hh)) : pl.k_base;
    const int k8_base = (n >> 4) * P::kTile + P::kRowBytes * r16 + 16 * ((swz(r16) & PUM) ^ hh);
    // e4m3: V through the transposing read of bytes: lane a of sixteen supplies row a / 2 of eight, keys 4 hh .. + 3 and 8 + 4 hh .. + 3
    const int va = lane & 15, vrow = 4 * hh + ((va >> 1) & 3) + 8 * (va >> 3);
    const int v8_base = P::kRowBytes * vrow + 16 * (((lane >> 4) & 1) ^ (swz(vrow) & PUM)) + 8 * (va & 1);

#pragma unroll 1
    for (int i = 0; i < mine; i++) {
        const int key = 32 * (t.lo + wave + kExWaves * i);
        const bool more = i + 1 < mine;
        wait_vmcnt<NV>(); // K is there (V of the stage, asked for after it, may not be)
        asm volatile("" ::: "memory");
        float sk0 = a.scale_log2, sk1 = a.scale_log2, sv0[NG], sv1[NG];
        if (FP8) {
            f32x4 w = *(const f32x4 *)(lds + X::kScales + 256 * wave);
            sk0 *= w[0], sk1 *= w[2];
            sk0 = sk0 == 0.f ? 1e-30f : sk0, sk1 = sk1 == 0.f ? 1e-30f : sk1; // (zero times the mask's -inf would be NaN)
#pragma unroll
            for (int g = 0; g < NG; g++) sv0[g] = w[1], sv1[g] = w[3];
        }
        bf16x8 kf[KS];
        if (FP8) {
#pragma unroll
            for (int k = 0; k < KS / 2; k++) {
                const uint4 c = *(const uint4 *)(lds + wave * X::kWave + (k8_base ^ (32 * k)));
                kf[2 * k] = fp8x8_to_bf16((int)c.x, (int)c.y), kf[2 * k + 1] = fp8x8_to_bf16((int)c.z, (int)c.w);
            }
        } else {
            uint32_t ka = k_addr + (uint32_t)pl.k_base;
            asm volatile("" : "+v"(ka));
#pragma unroll
            for (int k = 0; k < KS; k++) kf[k] = *(lds_bf16x8)(ka ^ (uint32_t)(32 * k));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) load_k(i + 1);
        const bool masked = key + 31 > first_lim;
        u32x4 pw[NG][2];
        // (two chains of products either way: of two groups of rows, or of one in halves)
        f32x16 sc[2];
#pragma unroll
        for (int e = 0; e < 16; e++) sc[0][e] = sc[1][e] = 0.f;
        uint32_t qa = q_addr + (uint32_t)kq_base;
        asm volatile("" : "+v"(qa));
#pragma unroll
        for (int k = 0; k < KS; k += 2) {
#pragma unroll
            for (int h = 0; h < 2; h++) {
                // (e4m3: unit 2 k + 2 hh + h; else 2 (k + h) + hh)
                const uint32_t at = qa ^ (uint32_t)(FP8 ? 32 * k + 16 * h : 32 * (k + h));
#pragma unroll
                for (int g = 0; g < NG; g++) {
                    f32x16 &x = sc[NG == 2 ? g : h];
                    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[k + h], *((lds_bf16x8)at + 2 * G::kTile * g / 16), x, 0, 0, 0);
                }
            }
        }
        if (NG == 1) sc[0] += sc[1];
        const bool odd_scale = FP8 && masked && ex_odd(sk0, sk1, sv0[0], sv1[0]);
        if (__builtin_expect(odd_scale, 0)) {
#pragma unroll
            for (int g = 0; g < NG; g++) {
                ex_scale_seen(sc[g], sk0, sk1, key, lim[g], hh);
                sv0[g] = key > lim[g] ? 1.f : sv0[g], sv1[g] = key + kPage > lim[g] ? 1.f : sv1[g];
            }
            sk0 = sk0 < INFINITY ? sk0 : 1.f, sk1 = sk1 < INFINITY ? sk1 : 1.f;
        }
#pragma unroll
        for (int g = 0; g < NG; g++) {
            f32x16 &s = sc[g];
            if (masked) {
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    if (key + 8 * (e / 4) + 4 * hh + (e % 4) > lim[g]) s[e] = -INFINITY;
                }
            }
            float m0 = max3(first_max(s[0], s[1]), s[2], s[3]), m1 = max3(first_max(s[8], s[9]), s[10], s[11]);
            m0 = max3(max3(m0, s[4], s[5]), s[6], s[7]), m1 = max3(max3(m1, s[12], s[13]), s[14], s[15]);
            float mn = fmaxf(m0 * sk0, m1 * sk1);
            const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mn), __float_as_uint(mn), false, false);
            mn = max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[1]));
            const bool grew = mn > m[g] + kPfSlack;
            if (__any(grew)) {
                mn = grew ? mn : m[g];
                const float alpha = __builtin_amdgcn_exp2f(m[g] - mn);
                m[g] = mn;
                l[g] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; dt++) o[g][dt] *= alpha;
            }
            float acc0 = 0.f, acc1 = 0.f;
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], e < 8 ? sk0 : sk1, -m[g]));
                float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], e < 8 ? sk0 : sk1, -m[g]));
                acc0 += w0, acc1 += w1;
                if (FP8) w0 *= e < 8 ? sv0[g] : sv1[g], w1 *= e < 8 ? sv0[g] : sv1[g];
                pw[g][e >> 3][(e >> 1) & 3] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{w0, w1}), bf16x2));
            }
            l[g] += acc0 + acc1;
        }
        if (more) wait_vmcnt<NK>(); // V is there
        else wait_vmcnt<0>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_setprio(1); // (as in ex_step: 64 drafts 79.8 -> 79.1 us)
        bf16x8 vf[DT][2];
        uint32_t vb = v_addr + (uint32_t)(FP8 ? v8_base : pl.v_base);
        asm volatile("" : "+v"(vb));
#pragma unroll
        for (int dt = 0; dt < DT; dt++) {
#pragma unroll
            for (int kk = 0; kk < 2; kk++) {
                if (FP8) {
                    const i32x2 c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(vb ^ (uint32_t)(32 * dt)) + kk * P::kTile / 8);
                    vf[dt][kk] = fp8x8_to_bf16(c[0], c[1]);
                } else {
                    const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb ^ (uint32_t)pf_v_xor<D>(dt, 0)) + kk * G::kTile / 8);
                    const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb ^ (uint32_t)pf_v_xor<D>(dt, 1)) + kk * G::kTile / 8);
                    vf[dt][kk] = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (more) load_v(i + 1);
        bool odd = false;
        if (masked) {
#pragma unroll
            for (int dt = 0; dt < DT; dt++) odd = odd || ex_odd(vf[dt][0]) || ex_odd(vf[dt][1]);
            odd = __any(odd);
        }
        if (__builtin_expect(odd, 0)) {
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
#pragma unroll
                for (int kk = 0; kk < 2; kk++) {
                    u32x4 plus, minus;
                    vf[dt][kk] = ex_even(vf[dt][kk], plus, minus);
#pragma unroll
                    for (int g = 0; g < NG; g++) {
                        const bf16x8 seen = ex_seen(key + 16 * kk, lim[g], hh);
                        ex_add_odd(o[g][dt], plus, seen, INFINITY), ex_add_odd(o[g][dt], minus, seen, -INFINITY);
                    }
                }
            }
        }
#pragma unroll
        for (int dt = 0; dt < DT; dt++) {
#pragma unroll
            for (int kk = 0; kk < 2; kk++) {
#pragma unroll
                for (int g = 0; g < NG; g++) o[g][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[dt][kk], __builtin_bit_cast(bf16x8, pw[g][kk]), o[g][dt], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    }

    // The waves' sums, 32 rows at a time, as the accumulators lie: 256 consecutive values (four of a lane) to a piece.
    constexpr int PIECES = 8; // of 32 rows and 64 d
    float2 *const stats = (float2 *)(lds + X::kStats);
#pragma unroll
    for (int g = 0; g < NG; g++) {
        const int row = t.row0 + 32 * g + n;
        float lg;
        {
            const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[g]), __float_as_uint(l[g]), false, false);
            lg = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
        const int token = ex_div_g(a, row < t.rows ? row : t.rows - 1);
        const int64_t rh = (int64_t)(p.s.t0 + token) * a.Hq + t.kvh * a.G + (row - token * a.G);
        float f[kExWaves], mm = kPfLowest, ll = 0.f, inv = 0.f;
#pragma unroll
        for (int half = 0; half < D / 64; half++) {
            __syncthreads(); // (nothing is on its way to the ring any more, and nothing of it is being read)
#pragma unroll
            for (int dt = 0; dt < 2; dt++) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const f32x16 &x = o[g][2 * half + dt];
                    *(f32x4 *)(lds + wave * X::kSum + 1024 * (4 * dt + j) + 16 * lane) = f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
                }
            }
            if (half == 0 && hh == 0) stats[32 * wave + n] = make_float2(m[g], lg);
            __syncthreads();
            if (half == 0) {
                float2 ml[kExWaves];
#pragma unroll
                for (int w = 0; w < kExWaves; w++) ml[w] = stats[32 * w + n], mm = fmaxf(mm, ml[w].x);
#pragma unroll
                for (int w = 0; w < kExWaves; w++) f[w] = __builtin_amdgcn_exp2f(ml[w].x - mm), ll += f[w] * ml[w].y;
                inv = ll > 0.f ? 1.0f / ll : ll == 0.f ? 0.f : ll; // (no key: zeros; NaN stays)
            }
#pragma unroll
            for (int x = 0; x < PIECES / kExWaves; x++) {
                const int c = PIECES / kExWaves * wave + x;
                f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kExWaves; w++) acc += f[w] * *(const f32x4 *)(lds + w * X::kSum + 1024 * c + 16 * lane);
                if (row >= t.rows) continue;
                if (t.slot >= 0) *(f32x4 *)(a.part_o + (int64_t)t.slot * (kExRows * D) + g * (32 * D) + 256 * (PIECES * half + c) + 4 * lane) = acc;
                else *(bf16x4 *)(a.out + rh * D + 64 * half + 32 * (c >> 2) + 8 * (c & 3) + 4 * hh) = __builtin_convertvector(acc * inv, bf16x4);
            }
        }
        if (wave == 0 && hh == 0 && row < t.rows) {
            if (t.slot >= 0) *(float2 *)(a.part_lse + 2 * ((int64_t)t.slot * kExRows + 32 * g + n)) = make_float2(mm, ll);
            else a.lse[rh] = (mm + __builtin_amdgcn_logf(ll)) * 0.6931471805599453f;
        }
    }
    __syncthreads(); // (the ring takes the next part's stages)
}

// The LDS of a workgroup: a ring of stages in bf16, and for each wave an area of its own, where e4m3 tiles land as they are
// stored (a ring of its own loads) and results are put in order on their way out.
template <int D, bool FP8> struct ExTileLds {
    static constexpr int kSlots = FP8 ? 3 : 4, kRaw = 3;
    static constexpr int kRawSlot = Geo<D, 1>::kTile + 256; // a tile, and the stage's scales
    static constexpr int kArea = FP8 && kRaw * kRawSlot > kPfStageBytes ? kRaw * kRawSlot : kPfStageBytes;
    static constexpr int kAreas = kSlots * Geo<D, 2>::kStage; // the areas follow the ring
    static constexpr int kBytes = kAreas + kArea * kExWaves;
    using N = ExNarrowLds<D, FP8>;
    static_assert(N::kNeeds <= kAreas && N::kRows <= kArea * kExWaves && N::kEnds <= kBytes, "few rows find room in it");
};

// What the rows of a kernel's sequences (of one kv head) are: any number; up to 32; up to 64; up to 32 or any number.  (64 drafts of
// 28 rows 59.8 us by kEx32, 91.3 by kExAny, e4m3 43.4 and 120; of 35 rows 79.1 by kEx64, 85.5, e4m3 60.1 and 68.0; for kExTwo see
// extend_shape.)
enum ExKind { kExAny, kEx32, kEx64, kExTwo };

template <int D, bool FP8, ExKind KIND> __global__ __launch_bounds__(64 * kExWaves, D == 64 ? 3 : 2) void extend_kernel(EX_PARAMS)
{
    EX_TAKE(a);
    using G = Geo<D, 2>;
    using P = Geo<D, FP8 ? 1 : 2>; // as the pools have it
    using X = ExTileLds<D, FP8>;
    extern __shared__ __attribute__((aligned(16384))) uint8_t lds[]; // the step forms LDS addresses by XOR
    const uint32_t lds_addr = (uint32_t)(uintptr_t)lds;
    const int lane = threadIdx.x & 63, n = lane & 31, hh = lane >> 5;
    const int wave = ex_uni((int)threadIdx.x >> 6);
    LaneConst<D, FP8 ? 1 : 2> lc;
    lane_setup<D, FP8 ? 1 : 2>(lc, lane, a.stride_token_b);
    PfLane<D> pl;
    pf_lane_setup<D>(pl, lane);
    uint8_t *const area = lds + X::kAreas + X::kArea * wave;
    const uint32_t area_addr = lds_addr + X::kAreas + X::kArea * wave;
    auto after = [](int slot) __attribute__((always_inline)) { return slot + 1 == X::kSlots ? 0 : slot + 1; };
    int slot0 = 0; // ring slot of the part's first stage; the others follow

    auto few = [&](const ExPlace &p, const ExPart &t) __attribute__((always_inline)) {
        ex_narrow<D, FP8, KIND == kEx64 ? 2 : 1>(a, p, t, lc, pl, lds, lds + X::kAreas, lane, wave);
    };
    auto many = [&](const ExPlace &p, const ExPart &t) __attribute__((always_inline)) {
        const int nst = t.hi - t.lo, row = t.row0 + kPfRows * wave + n; // this lane's row
        const bool exists = row < t.rows;
        const int token = ex_div_g(a, exists ? row : t.rows - 1), head = t.kvh * a.G + ((exists ? row : t.rows - 1) - token * a.G);
        const int shift = p.s.L - p.s.n, lim = shift + token;
        // the wave's first and last row: stages below `whole` are seen by all of its rows, those from `mine` on by none
        const int row_lo = t.row0 + kPfRows * wave, row_hi = row_lo + kPfRows < t.rows ? row_lo + kPfRows - 1 : t.rows - 1;
        const int whole = row_lo < t.rows ? ex_uni((shift + ex_div_g(a, row_lo) + 1) >> 5) : 0;
        int mine = row_lo < t.rows ? ex_uni((shift + ex_div_g(a, row_hi) + 32) >> 5) : 0;
        mine = (mine < t.hi ? mine : t.hi) - t.lo; // of the part's stages

        // Wave w brings tile w of every stage (K of its two pages, V of its two pages).
        const int32_t *const pages = a.table + (int64_t)p.b * a.max_pages;
        const int count = (p.s.L + kPage - 1) / kPage; // pages that exist
        const int of = wave & 1; // the wave's page of a stage's two
        const uint8_t *const pool = (wave < 2 ? a.k_pool : a.v_pool) + (int64_t)t.kvh * a.stride_head_b;
        // (An id is asked for a stage ahead of its use, and looked at only there: until then the load may be on its way.  A page
        // that does not exist takes another's place in the row, or the first, and none of its rows are read.)
        const int last_page = count > 0 ? count - 1 : 0;
        auto page_id = [&](int s, int h) __attribute__((always_inline)) { // of page h of stage s of the part
            const int i = 2 * (t.lo + s) + h;
            return uniform_load(pages, i < last_page ? i : last_page);
        };
        int issued = 0, id = 0, other = 0;
        if (count > 0) {
            id = page_id(0, of);
            if (FP8) other = page_id(0, 1 - of);
        }
        int load_slot = FP8 ? 0 : slot0; // where the next tile goes (e4m3: in the wave's own ring)
        constexpr int DPW = P::kDmaPerTile + (FP8 ? 1 : 0); // a wave's loads per stage
        auto issue = [&]() __attribute__((always_inline)) { // the next stage's tile
            if (issued >= nst) return;
            const int valid = p.s.L - kPage * (2 * (t.lo + issued) + of);
            const uint32_t to = FP8 ? area_addr + load_slot * X::kRawSlot : lds_addr + load_slot * G::kStage + wave * G::kTile;
            issue_tile<D, FP8 ? 1 : 2>(lc, pool + (int64_t)id * a.stride_page_b, valid, to, a.zeros);
            if (FP8) { // lanes 0..3 bring K and V scale of the first page, K and V scale of the second
                const int h = (lane >> 1) & 1, pid = h == of ? id : other;
                const void *src = a.zeros;
                if (lane < 4 && (h == of ? valid : p.s.L - kPage * (2 * (t.lo + issued) + 1 - of)) > 0)
                    src = ((lane & 1) ? a.v_scale : a.k_scale) + (int64_t)pid * a.Hkv + t.kvh;
                dma4(src, to + P::kTile);
            }
            issued++;
            load_slot = FP8 ? (load_slot + 1 == X::kRaw ? 0 : load_slot + 1) : after(load_slot);
            id = page_id(issued, of);
            if (FP8) other = page_id(issued, 1 - of);
        };
        ExScale sc = {a.scale_log2, a.scale_log2, 1.f, 1.f}, sc_next = sc, sc_put = sc;
        int raw_slot = 0, put_slot = slot0;
        // e4m3 pools: the wave's tile of stage s, once landed, goes into the ring as bf16 (exactly; its scales stay apart)
        auto put = [&](int s) __attribute__((always_inline)) {
            WaitTail<X::kRaw - 1, DPW>::run(issued - 1 - s);
            asm volatile("" ::: "memory");
            const uint8_t *const from = area + raw_slot * X::kRawSlot;
            uint8_t *const tile = lds + put_slot * G::kStage + wave * G::kTile;
            const f32x4 w = *(const f32x4 *)(from + P::kTile);
            uint4 raw[P::kDmaPerTile];
#pragma unroll
            for (int x = 0; x < P::kDmaPerTile; x++) raw[x] = *(const uint4 *)(from + 1024 * x + 16 * lane);
#pragma unroll
            for (int x = 0; x < P::kDmaPerTile; x++) {
                const int u = 64 * x + lane, r = u / P::kUnits, c = (u % P::kUnits) ^ (swz(r) & (P::kUnits - 1)), z = swz(r) & (G::kUnits - 1);
                *(bf16x8 *)(tile + 16 * (r * G::kUnits + ((2 * c) ^ z))) = fp8x8_to_bf16((int)raw[x].x, (int)raw[x].y);
                *(bf16x8 *)(tile + 16 * (r * G::kUnits + ((2 * c + 1) ^ z))) = fp8x8_to_bf16((int)raw[x].z, (int)raw[x].w);
            }
            auto scale = [&](float f, bool k) __attribute__((always_inline)) {
                const int bits = ex_uni(__float_as_int(f));
                return __int_as_float(k && (bits & 0x7fffffff) == 0 ? 0x0da24260 : bits); // (1e-30: zero times the mask's -inf would be NaN)
            };
            sc_put = {scale(w[0] * a.scale_log2, true), scale(w[2] * a.scale_log2, true), scale(w[1], false), scale(w[3], false)};
            raw_slot = raw_slot + 1 == X::kRaw ? 0 : raw_slot + 1;
            put_slot = after(put_slot);
        };
        // Before the first step that reads stage s: it has landed, for every wave, and every wave has left the step that read
        // stage s - 2, whose slot the next load (e4m3: stage s + 1) may take.
        auto open = [&](int s) __attribute__((always_inline)) {
            if (!FP8) WaitTail<X::kSlots - 1, DPW>::run(issued - 1 - s);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (FP8) {
                sc = sc_next, sc_next = sc_put;
                if (s + 1 < nst) put(s + 1);
            }
            issue();
        };

        PfState<D> st;
        {
            const uint16_t *const q = a.q + (int64_t)(p.s.t0 + token) * a.q_stride + head * D + 8 * hh;
#pragma unroll
            for (int i = 0; i < D / 16; i++) st.qf[i] = *(const bf16x8 *)(q + 16 * i);
        }
        // (the barriers of the part before have passed the slots that are filled now)
        issue();
        issue();
        if (FP8) {
            issue();
            if (nst > 0) put(0);
        }
        st.m = kPfLowest, st.lsum = 0.f;
#pragma unroll
        for (int dt = 0; dt < D / 32; dt++) {
#pragma unroll
            for (int e = 0; e < 16; e++) st.o[dt][e] = 0.f;
        }
        // Stage s is opened before step s - 1, which makes its scores; the first one before the scores alone.
        if (nst > 0) {
            open(0);
            if (FP8) sc = sc_next; // (stage 0; sc_next: stage 1 once that has been opened)
            if (mine > 0) {
                pf_scores<D>(lds_addr + slot0 * G::kStage, pl, st.qf, st.s);
                if (t.lo >= whole) {
#pragma unroll
                    for (int e = 0; e < 16; e++) {
                        if (32 * t.lo + 8 * (e / 4) + 4 * hh + (e % 4) > lim) st.s[e] = -INFINITY;
                    }
                }
                float m0 = first_max(st.s[0], st.s[1]), m1 = first_max(st.s[8], st.s[9]);
#pragma unroll
                for (int e = 2; e < 8; e += 2) m0 = max3(m0, st.s[e], st.s[e + 1]), m1 = max3(m1, st.s[8 + e], st.s[9 + e]);
                float mx = fmaxf(m0 * sc.k0, m1 * sc.k1);
                const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                st.m = fmaxf(max3(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[1])), kPfLowest);
            }
            int cur = slot0, nxt = after(slot0); // of stages s and s + 1
#define EX_STEP(MASK, NEXT)                                                                                                          \
    ex_step<D, FP8, MASK, NEXT>(st, lds_addr + nxt * G::kStage, lds_addr + cur * G::kStage + 2 * G::kTile, pl, sc, sc_next, 32 * (t.lo + s), \
                                32 * (t.lo + s + 1), lim);                                                                            \
    cur = nxt, nxt = after(nxt)
            int s = 0;
            auto advance = [&]() __attribute__((always_inline)) {
                if (s + 1 < nst) open(s + 1);
                else if (FP8) sc = sc_next;
            };
            if (mine > 0) {
                const int free = whole - t.lo < mine ? whole - t.lo : mine; // stages without a mask
                // (two steps at a time: the scores need not change registers)
#pragma unroll 1
                for (; s + 2 < free; s++) {
                    open(s + 1);
                    EX_STEP(false, true);
                    s++;
                    open(s + 1);
                    EX_STEP(false, true);
                }
                if (s + 1 < free) {
                    open(s + 1);
                    EX_STEP(false, true);
                    s++;
                }
#pragma unroll 1
                for (; s + 1 < mine; s++) {
                    open(s + 1);
                    EX_STEP(true, true);
                }
                advance();
                EX_STEP(false, false);
                s++;
            }
            for (; s < nst; s++) advance();
#undef EX_STEP
            slot0 = ex_uni((slot0 + nst) % X::kSlots);
        }

        // a row's sum is spread over its two lanes
        float l;
        {
            const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.lsum), __float_as_uint(st.lsum), false, false);
            l = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }
        if (row_lo >= t.rows) return;
        if (t.slot >= 0) {
            // a part: as the accumulators lie, which is whole lines
            float *const o = a.part_o + (int64_t)t.slot * (kExRows * D) + wave * (kPfRows * D) + 4 * lane;
#pragma unroll
            for (int dt = 0; dt < D / 32; dt++) {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (exists) *(f32x4 *)(o + 256 * (4 * dt + j)) = f32x4{st.o[dt][4 * j], st.o[dt][4 * j + 1], st.o[dt][4 * j + 2], st.o[dt][4 * j + 3]};
            }
            if (exists && hh == 0) *(float2 *)(a.part_lse + 2 * ((int64_t)t.slot * kExRows + kPfRows * wave + n)) = make_float2(st.m, l);
            return;
        }
        const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l; // (no key: zeros; NaN stays)
#pragma unroll
        for (int pc = 0; pc < D / 64; pc++) {
#pragma unroll
            for (int dtl = 0; dtl < 2; dtl++) {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    f32x4 v;
#pragma unroll
                    for (int x = 0; x < 4; x++) v[x] = st.o[2 * pc + dtl][4 * j + x] * inv;
                    *(bf16x4 *)(area + kPfStageRow * n + 16 * ((4 * dtl + j) ^ pf_stage_swz(n)) + 8 * hh) = __builtin_convertvector(v, bf16x4);
                }
            }
#pragma unroll
            for (int m = 0; m < 4; m++) {
                const int r = 8 * m + (lane >> 3), c = lane & 7, orow = row_lo + r;
                const u32x4 v = *(const u32x4 *)(area + kPfStageRow * r + 16 * (c ^ pf_stage_swz(r)));
                if (orow < t.rows) {
                    const int i = ex_div_g(a, orow);
                    *(u32x4 *)(a.out + ((int64_t)(p.s.t0 + i) * a.Hq + t.kvh * a.G + (orow - i * a.G)) * D + 64 * pc + 8 * c) = v;
                }
            }
        }
        if (exists && hh == 0) a.lse[(int64_t)(p.s.t0 + token) * a.Hq + head] = (st.m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    };
    if constexpr (KIND == kExTwo) ex_walk<true>(a, lds, many, few);
    else if constexpr (KIND == kExAny) ex_walk<false>(a, lds, many, many);
    else ex_walk<false>(a, lds, few, few);
    wait_vmcnt<0>(); // nothing may land in LDS after the workgroup has left
}

// ---- what spans share -----------------------------------------------------------------------------------

constexpr int kExMaxSpans = 1024, kExMergeWgs = 4; // workgroups of the merge for each span
constexpr int kExMergeFew = 12; // an item of fewer parts is one wave's to add up (one of 64 parts: 47.3 us in all, so too 55.4; all
                                // items by four waves: 64 drafts 85.6 us, so 79.1)

// Adds up the parts of the items that a cut goes through, 256 consecutive values of an item's parts at a time.  An item of P
// parts lies in P - 1 spans that begin inside it: each of them has every (P - 1)-th of the item's chunks of 256 values to add
// up, so that all have as much to read.  Its time is the launch, two trips and the parts: 7 us for 64
// drafts (15 MB read), 8 for a mixed batch (24 MB), 9 for 96 short turns (31 MB), 4 where there are none.  A wave does so alone where the item has few parts, else a workgroup's waves take
// every fourth part each.
template <int D> __global__ __launch_bounds__(64 * kExWaves) void extend_merge_kernel(const int4 *__restrict__ desc, ExtendLaunch given)
{
    ExtendLaunch a = given;
    touch_lines(given);
    constexpr int W = kExWaves, GROUP = D / 8; // chunks of 32 rows
    __shared__ f32x4 sums[W][64];
    __shared__ float2 stats[W][64];
    const int lane = threadIdx.x & 63, wave = ex_uni((int)threadIdx.x >> 6);
    const int j = blockIdx.x / kExMergeWgs, sub = blockIdx.x % kExMergeWgs;
    const int4 item = desc[2 * j], ends = desc[2 * j + 1];
    const int k = ex_uni(ends.x), last = ex_uni(ends.y);
    if (k < 0) return;
    const int left = ex_uni(item.z - item.y), chunks = left >= kExRows ? GROUP * kExWaves : GROUP * ((left + 31) >> 5);
    const bool split = last - k + 1 >= kExMergeFew;
    const int share = last - k; // spans with a share of the item
    for (int c0 = j - k - 1 + share * (split ? sub : W * sub); c0 < chunks; c0 += share * (split ? kExMergeWgs : W * kExMergeWgs)) {
        const int chunk = split ? c0 : c0 + share * wave;
        const bool have = chunk < chunks;
        int r, d; // this lane's row of the block, and the first of its four values
        {
            const int wv = chunk / (D / 8), c = chunk % (D / 8);
            r = kPfRows * wv + (lane & 31), d = 32 * (c >> 2) + 8 * (c & 3) + 4 * (lane >> 5);
        }
        const int row = item.y + r;
        const bool exists = have && row < item.z;
        float mm = kPfLowest, l = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        if (exists) {
            constexpr int AT = 4;
            const int step = split ? W : 1;
            for (int p0 = split ? k + wave : k; p0 <= last; p0 += AT * step) {
                float2 ml[AT];
                f32x4 o[AT];
#pragma unroll
                for (int i = 0; i < AT; i++) {
                    const int p = p0 + step * i;
                    const int64_t slot = p == k ? 2 * (int64_t)k + 1 : 2 * (int64_t)p;
                    ml[i] = make_float2(kPfLowest, 0.f), o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (p <= last) {
                        ml[i] = *(const float2 *)(a.part_lse + 2 * (slot * kExRows + r));
                        o[i] = *(const f32x4 *)(a.part_o + slot * (kExRows * D) + 256 * chunk + 4 * lane);
                    }
                }
                float top = mm;
#pragma unroll
                for (int i = 0; i < AT; i++) top = fmaxf(top, ml[i].x);
                const float f0 = __builtin_amdgcn_exp2f(mm - top);
                l *= f0, acc *= f0, mm = top;
#pragma unroll
                for (int i = 0; i < AT; i++) {
                    const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
                    l += f * ml[i].y, acc += f * o[i];
                }
            }
        }
        if (split) {
            sums[wave][lane] = acc, stats[wave][lane] = make_float2(mm, l);
            __syncthreads();
            mm = kPfLowest, l = 0.f, acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; w++) mm = fmaxf(mm, stats[w][lane].x);
#pragma unroll
            for (int w = 0; w < W; w++) {
                const float f = __builtin_amdgcn_exp2f(stats[w][lane].x - mm);
                l += f * stats[w][lane].y, acc += f * sums[w][lane];
            }
            __syncthreads();
        }
        if (exists && (wave == 0 || !split)) {
            const int token = ex_div_g(a, row);
            const int64_t rh = (int64_t)(item.x + token) * a.Hq + item.w * a.G + (row - token * a.G);
            const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
            *(bf16x4 *)(a.out + rh * D + d) = __builtin_convertvector(acc * inv, bf16x4);
            if (d == 0) a.lse[rh] = (mm + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
        }
    }
}

} // namespace ra
