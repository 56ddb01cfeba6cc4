// gfx950 kernels of the attention of chunks of new tokens over the paged cache.
//
// A sequence's n new tokens and the G query heads of a kv head are n * G rows that read the same keys: row r is token r / G,
// head r % G, and sees the keys up to L - n + r / G.  Packed that way 32 rows are a few tokens, so under the causal mask
// they need the same keys but for the last one or two stages of 32.
//
// Many rows are bound by the matrix cores: extend_tile_kernel, whose workgroup takes a block of 128 rows, 32 to a wave, all
// waves multiplying every stage of 32 keys that streams through one LDS ring:
//   S^T[key, row] = K . Q^T,   O^T[d, row] += V^T . P^T     (32x32x16 MFMA, binary32 sums, softmax running per row)
// Few rows are bound by the stream of pages: extend_few_kernel, whose four waves stream stages of their own (every fourth
// one) through rings of their own and multiply them with all of the up to 32 rows; what they have is added up in LDS.
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
constexpr int kExTileRows = kPfRows * kExWaves; // rows of a block of the tile kernel
constexpr int kExFewRows = 32;                  // rows of a sequence and kv head up to which the other one takes them

// ---- the line of items and its spans ------------------------------------------------------------------

struct ExSeq {
    int t0, n, L;  // first packed token, new tokens, tokens in all
    int blocks, cost; // blocks of a kv head; the length of each on the line (stages, the mean of the sequence's blocks, and kFixed)
};

// What an item costs beside its stages, in stages: finding it, its query rows, the first trip to memory, its results.
template <int ROWS> constexpr int kExFixed = ROWS == kExTileRows ? 4 : 8;
constexpr int kExEdge = 2; // no part of an item has fewer stages than this (about; a span is longer than kExFixed + 2 kExEdge)

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
template <int ROWS> __device__ __forceinline__ int ex_stages(const ExtendLaunch &a, const ExSeq &s, int j)
{
    int last = ex_div_g(a, ROWS * (j + 1) - 1);
    last = s.L - s.n + (last < s.n - 1 ? last : s.n - 1);
    return (last + 32) >> 5; // (last >= -n: no key at all gives a number of zero or less)
}
// ... where x is often below 64 y: the multiples of y up to x are counted.
__device__ __forceinline__ int ex_div_short(int x, int y)
{
    if (x >= 64 * y) return ex_div(x, y);
    return __popcll(__ballot((int)(threadIdx.x & 63) * y <= x)) - 1;
}

// What the sequence of t0, t1 (where its chunk starts and ends) and length L is.  (A workgroup comes past everything up to its
// first keys once and alone, an instruction after the other: they are few.)
template <int ROWS> __device__ __forceinline__ ExSeq ex_sequence(const ExtendLaunch &a, int t0, int t1, int L)
{
    ExSeq s = {0, 0, 0, 0, 0};
    const int n = t1 - t0, most = a.max_pages * kPage;
    if (t0 < 0 || t0 > a.T || n <= 0 || n > a.T - t0) return s;
    s.t0 = t0;
    s.n = n < a.max_chunk ? n : a.max_chunk;
    s.L = L < 0 ? 0 : (L < most ? L : most);
    s.blocks = (s.n * a.G + ROWS - 1) / ROWS;
    const int mean = (s.L - (s.n >> 1) + 48) >> 5; // keys that a row sees, in stages
    s.cost = kExFixed<ROWS> + (mean > 1 ? mean : 1);
    return s;
}
template <int ROWS> __device__ __forceinline__ ExSeq ex_sequence(const ExtendLaunch &a, int b)
{
    return b < a.B ? ex_sequence<ROWS>(a, a.cu[b], a.cu[b + 1], a.seq_lens[b]) : ExSeq{0, 0, 0, 0, 0};
}

// The line: lane c has chunk c of the sequences (64 of them, or a multiple of that in a very large batch).  Of a batch of up to
// 512, `known` keeps in LDS what the first search for a place needs; every wave writes all of it, the same values to the same
// place.
constexpr int kExKnown = 512;
struct ExKnown {
    int4 rec[kExKnown]; // {start on the line, blocks before, first packed token, new tokens}
    int len[kExKnown];
};
static_assert(sizeof(ExKnown) <= 3 * Geo<64, 2>::kStage, "it fits the smallest ring");

template <int ROWS> struct ExLine {
    int lane, sub, chunks;   // sixty-fours of sequences in a chunk
    int unit;                // items are left whole (see measure)
    int before, total;       // start of this lane's chunk
    int before_blocks, blocks; // ... counted in blocks of one kv head
    int q, r, spans, cut;    // span k starts at q k + min(k, r), before cuts are moved; items up to `cut` are not cut

    __device__ __forceinline__ void measure(const ExtendLaunch &a, ExKnown *known)
    {
        lane = threadIdx.x & 63;
        before = before_blocks = total = blocks = 0;
        int longest = 0;
        sub = 1;
        auto add = [&](const ExSeq &s, int &at, int &at_blocks) __attribute__((always_inline)) {
            int tc, tb;
            at = total + wave_scan(a.Hkv * s.blocks * s.cost, lane, tc), at_blocks = blocks + wave_scan(s.blocks, lane, tb);
            total += tc, blocks += tb;
            longest = longest > s.cost ? longest : s.cost;
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
                    const ExSeq s = ex_sequence<ROWS>(a, t0[i], t1[i], len[i]);
                    if (lane == c0 + i) before = total, before_blocks = blocks;
                    int at, at_blocks;
                    add(s, at, at_blocks);
                    known->rec[64 * (c0 + i) + lane] = make_int4(at, at_blocks, s.t0, s.n);
                    known->len[64 * (c0 + i) + lane] = s.L;
                }
            }
        } else {
            sub = (a.B + 4095) >> 12;
            chunks = ex_div(a.B + 64 * sub - 1, 64 * sub);
#pragma unroll 1
            for (int c = 0; c < chunks * sub; c++) {
                if (lane * sub == c) before = total, before_blocks = blocks;
                int at, at_blocks;
                add(ex_sequence<ROWS>(a, 64 * c + lane), at, at_blocks);
            }
        }
        if (lane >= chunks) before = before_blocks = INT32_MAX;
        spans = a.spans;
        if (total < a.least * a.spans) {
            spans = ex_div(total, a.least);
            spans = spans < 1 ? 1 : spans;
        }
        q = ex_div(total, spans);
        r = total - q * spans;
        cut = q >> 3 > a.cut ? q >> 3 : a.cut;
        // Many items, none of them longer than what a workgroup has on average: they are left whole, a workgroup for each.
        unit = blocks * a.Hkv >= 2 * a.spans && !__any(longest > q);
    }
    __device__ __forceinline__ int raw(int k) const { return q * k + (k < r ? k : r); }
    // The last span that an item which ends at x1 has a part in, if it is cut.
    __device__ __forceinline__ int last_of(int x1) const
    {
        const int y = x1 - 1, big = r * (q + 1);
        const bool in_big = y < big;
        const int k = (in_big ? 0 : r) + ex_div(in_big ? y : y - big, in_big ? q + 1 : q); // the last one that starts before x1
        return x1 - raw(k) < kExEdge ? k - 1 : k;                          // (but for a cut that moves there)
    }
    // Where a cut at x goes in the item of that length that starts at x0: nowhere into short items, and not so near an end of
    // others that a part would be next to nothing.
    __device__ __forceinline__ int moved(int x, int x0, int cost) const
    {
        const int y = x - x0, left = cost - y;
        const bool down = cost > cut ? y < kExFixed<ROWS> + kExEdge : y < left, up = cost > cut ? left < kExEdge : true;
        return down ? x0 : up ? x0 + cost : x;
    }
};

// A place on the line: an item of a sequence.
struct ExPlace {
    int b, item, x0; // the sequence, its item (kv head * blocks + number), the item's start
    ExSeq s;         // (cost: the item's length on the line)
};

// The sequence that x lies in (0 <= x < total), x counted as the line is or (BLOCKS) in blocks of one kv head; returns x's
// distance from its start.
template <int ROWS, bool BLOCKS> __device__ __forceinline__ int ex_sequence_at(const ExtendLaunch &a, const ExLine<ROWS> &line, const ExKnown *known, int x, ExPlace &p)
{
    const int chunk_before = BLOCKS ? line.before_blocks : line.before;
    const int c = 63 - __builtin_clzll(__ballot(chunk_before <= x));
    int base = 64 * c, before;
    ExSeq s = {0, 0, 0, 0, 0};
    if (known) {
        const int4 rec = known->rec[base + line.lane];
        s.t0 = rec.z, s.n = rec.w, s.L = known->len[base + line.lane], before = BLOCKS ? rec.y : rec.x;
    } else {
        int start = __builtin_amdgcn_readlane(chunk_before, c);
#pragma unroll 1
        for (int i = 0;; i++) {
            base = (c * line.sub + i) * 64;
            s = ex_sequence<ROWS>(a, base + line.lane);
            int t;
            before = start + wave_scan(BLOCKS ? s.blocks : a.Hkv * s.blocks * s.cost, line.lane, t);
            if (x < start + t || i + 1 == line.sub) break;
            start += t;
        }
    }
    const int l = 63 - __builtin_clzll(__ballot(s.n > 0 && before <= x));
    p.b = base + l;
    const int t0 = __builtin_amdgcn_readlane(s.t0, l);
    p.s = ex_sequence<ROWS>(a, t0, t0 + __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.L, l));
    return x - __builtin_amdgcn_readlane(before, l);
}

// The item that x lies in.
template <int ROWS> __device__ __forceinline__ void ex_find(const ExtendLaunch &a, const ExLine<ROWS> &line, const ExKnown *known, int x, ExPlace &p)
{
    const int y = ex_sequence_at<ROWS, false>(a, line, known, x, p);
    p.item = ex_div_short(y, p.s.cost);
    p.x0 = x - y + p.item * p.s.cost;
}

// A part of an item that a workgroup works on.
struct ExPart {
    int kvh, row0, rows; // rows of the sequence and kv head in all
    int lo, hi;          // stages
    int slot;            // -1: the item is whole; else where its part goes
};

// The blocks of a (sequence, kv head) come from both ends in turn: their mean cost is the line's.
template <int ROWS> __device__ __forceinline__ ExPart ex_part(const ExtendLaunch &a, const ExPlace &p, int y0, int y1, int span)
{
    ExPart t;
    t.kvh = ex_div_short(p.item, p.s.blocks);
    const int jj = p.item - t.kvh * p.s.blocks, j = jj & 1 ? p.s.blocks - 1 - (jj >> 1) : jj >> 1;
    t.row0 = ROWS * j;
    t.rows = p.s.n * a.G;
    int stages = ex_uni(ex_stages<ROWS>(a, p.s, j));
    stages = stages < 0 ? 0 : stages;
    // (a place inside the item, in proportion: the same for the two parts that it divides)
    auto stage_at = [&](int y) __attribute__((always_inline)) {
        return ex_uni((int)((float)stages * ((float)(y - kExFixed<ROWS>) * __builtin_amdgcn_rcpf((float)(p.s.cost - kExFixed<ROWS>)))));
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
// Else: a die takes neighbouring spans.  Also tells the merge which items begin in a span and end in another: desc[2 k],
// desc[2 k + 1] = {first packed token, first row, rows, kv head}, {last span, -, -, -}.
template <int ROWS, typename F> __device__ __forceinline__ void ex_walk(const ExtendLaunch &a, uint8_t *lds, F &&work)
{
    const int die = (int)blockIdx.x & 7, at = (int)blockIdx.x >> 3;
    const int gg_shift = (a.Hkv & 7) == 0 ? 3 : (a.Hkv & 3) == 0 ? 2 : (a.Hkv & 1) == 0 ? 1 : 0, s_shift = 3 - gg_shift, heads = a.Hkv >> gg_shift;
    const int first_head = die & ((1 << gg_shift) - 1), share = (at << s_shift) + (die >> gg_shift);
    const ExKnown *known = a.B <= kExKnown ? (ExKnown *)lds : nullptr;
    ExLine<ROWS> line;
    ExPlace p;
    ExPart part;
    p.item = 0, p.x0 = 0;
    int last = 0, x = 0, end = 0, step = 0, k = 0;
    int4 begun = {0, 0, 0, 0};
    if (a.direct) {
        // Every item is short: a workgroup for each, and no line.  Blocks are numbered without counting them: sequence b's
        // are given the numbers from cu[b] G / ROWS + b on, which leaves it as many as it can have.
        const int number = ex_div_short(share, heads), lane = threadIdx.x & 63;
        int j = 0;
        p.b = number;
        if (ROWS != kExFewRows) { // (few rows are one block)
            p.b = -1;
#pragma unroll 1
            for (int base = 0; base < a.B; base += 64) {
                const int start = base + lane < a.B ? (int)((int64_t)a.cu[base + lane] * a.G / ROWS) + base + lane : INT32_MAX;
                const unsigned long long m = __ballot(start <= number);
                if (!m) break;
                const int l = 63 - __builtin_clzll(m);
                p.b = base + l, j = number - __builtin_amdgcn_readlane(start, l);
                if (l < 63) break;
            }
        }
        if (p.b < 0 || p.b >= a.B) return;
        p.s = ex_sequence<ROWS>(a, uniform_load(a.cu, p.b), uniform_load(a.cu, p.b + 1), uniform_load(a.seq_lens, p.b));
        if (j < 0 || j >= p.s.blocks) return;
        part.kvh = ((share - number * heads) << gg_shift) + first_head;
        part.row0 = ROWS * j, part.rows = p.s.n * a.G;
        part.lo = 0, part.hi = ex_stages<ROWS>(a, p.s, j), part.slot = -1;
        part.hi = part.hi < 0 ? 0 : part.hi;
        end = 1;
    } else {
        line.measure(a, (ExKnown *)lds);
        const int per = (line.spans + 7) >> 3;
        k = at < per ? die * per + at : (int)blockIdx.x; // (past the spans: one that does not exist)
        if (line.unit) {
            x = share, end = line.blocks * heads;
            step = (int)gridDim.x >> 3 << s_shift; // (there are as many workgroups as items, if the call's sizes are what they say)
        } else if (line.total > 0 && at < per && k < line.spans) {
            // `end` is moved where the span gets to it
            end = k + 1 < line.spans ? line.raw(k + 1) : line.total, x = line.raw(k);
            ex_find<ROWS>(a, line, known, x, p);
            x = line.moved(x, p.x0, p.s.cost);
            if (x == p.x0 + p.s.cost) {
                if (p.item + 1 < a.Hkv * p.s.blocks) p.item++, p.x0 = x;
                else if (x < end) ex_find<ROWS>(a, line, known, x, p);
            }
        }
    }
    bool first = !a.direct;
    while (x < end) {
        int next = 1;
        if (a.direct) {
        } else if (line.unit) {
            const int at_block = ex_div(x, heads);
            const int i = x - (at_block - ex_sequence_at<ROWS, true>(a, line, first ? known : nullptr, at_block, p)) * heads;
            const int h = ex_div_short(i, p.s.blocks); // (a sequence's items: its blocks times heads)
            p.item = i + ((h << gg_shift) + first_head - h) * p.s.blocks;
            part = ex_part<ROWS>(a, p, 0, p.s.cost, 0);
            next = x + step;
        } else {
            const int x1 = p.x0 + p.s.cost;
            if (end < x1) end = line.moved(end, p.x0, p.s.cost);
            if (x >= end) break;
            next = x1 < end ? x1 : end;
            part = ex_part<ROWS>(a, p, x - p.x0, next - p.x0, k);
            if (x == p.x0 && next < x1) {
                begun = make_int4(p.s.t0, part.row0, part.rows, part.kvh);
                last = line.last_of(x1);
            }
        }
        if (first) __syncthreads(); // (what the waves know of the line makes room for the ring)
        first = false;
        work(p, part);
        x = next;
        if (x >= end || line.unit) continue;
        if (p.item + 1 < a.Hkv * p.s.blocks) p.item++, p.x0 = x;
        else ex_find<ROWS>(a, line, nullptr, x, p);
    }
    if (threadIdx.x == 0 && !a.direct && k < a.spans) { // (every span is answered for, also one that does not exist)
        a.desc[2 * k] = begun;
        a.desc[2 * k + 1] = make_int4(last, 0, 0, 0);
    }
}

// ---- values that a row does not see ---------------------------------------------------------------------
//
// In the stages that the causal mask cuts, a row's weight of a later token is zero, and zero times an infinite or NaN value
// is NaN.  Where a V operand of such a stage holds one, its product is made key by key, each added only to rows that see it.

__device__ __forceinline__ bool ex_odd(bf16x8 v)
{
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 4; i++) odd = odd || (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
    return odd;
}
// The operand with only element e of its eight kept.
__device__ __forceinline__ bf16x8 ex_only(bf16x8 v, bool lanes, int e)
{
    u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] &= lanes && (e >> 1) == i ? 0xffffu << (16 * (e & 1)) : 0u;
    return __builtin_bit_cast(bf16x8, w);
}

// ---- many rows ------------------------------------------------------------------------------------------

// Scale of a stage's first and second page for the scores (softmax scale and binary logarithm included), and for V.
struct ExScale {
    float k0, k1, v0, v1;
};

// One step of a wave's software pipeline: the weights of a stage (whose scores are st.s) and the scores of the next
// (NEXT; MASK: the causal mask cuts one of the two), then O += P V of the first and the maxima of the new scores.
// key, key_next: first keys of the two stages; lim: the last key that the lane's row sees.
// As pf_step, but for the scales of e4m3 pages (their codes lie in the ring as bf16, exactly) and what MASK does with V.
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
    u32x4 pw[2];
    float pprev = 0.f, acc0 = 0.f, acc1 = 0.f;
    auto w_item = [&](int k) {
        if (k < 16) {
            float pk = __builtin_amdgcn_exp2f(__builtin_fmaf(st.s[k], k < 8 ? sc.k0 : sc.k1, -st.m));
            if (k & 1) acc1 = k == 1 ? pk : acc1 + pk;
            else acc0 = k == 0 ? pk : acc0 + pk;
            if (FP8) pk *= k < 8 ? sc.v0 : sc.v1;
            if (k & 1) pw[k >> 3][(k >> 1) & 3] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2{pprev, pk}), bf16x2));
            else pprev = pk;
        } else {
            st.lsum += acc0 + acc1;
        }
    };
    constexpr int NW = 17;
    f32x16 sn;
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
        else if (k == 10) mx = fmaxf(mx0 * sn_.k0, mx * sn_.k1);
        else if (k >= 12) m_item(k);
    };
    constexpr int NMI = NEXT ? 14 : 0, NPV = 2 * DT;
#pragma unroll
    for (int n = 0; n < NPV; n++) {
        const int dt = n / 2, kk = n % 2;
        if (n + DT < NPV) v_read((n + DT) / 2, (n + DT) % 2);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(vr[dt][kk][0], vr[dt][kk][1], 0, 1, 2, 3, 4, 5, 6, 7));
        const bf16x8 pf = __builtin_bit_cast(bf16x8, pw[kk]);
        if ((MASK || !NEXT) && __builtin_expect(__any(ex_odd(vf)), 0)) {
#pragma unroll 1
            for (int i = 0; i < 16; i++) { // key 8 (e / 4) + 4 h + e % 4 of the sixteen: element e of the lanes of half h
                const int e = i & 7, h = i >> 3;
                f32x16 t;
#pragma unroll
                for (int x = 0; x < 16; x++) t[x] = 0.f;
                t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ex_only(vf, hh == h, e), pf, t, 0, 0, 0);
                const bool sees = key + 16 * kk + 8 * (e >> 2) + 4 * h + (e & 3) <= lim;
#pragma unroll
                for (int x = 0; x < 16; x++) st.o[dt][x] += sees ? t[x] : 0.f;
            }
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

// The LDS of a workgroup: a ring of stages in bf16, and for each wave an area of its own, where e4m3 tiles land as they are
// stored (a ring of its own loads) and results are put in order on their way out.
template <int D, bool FP8> struct ExTileLds {
    static constexpr int kSlots = FP8 ? 3 : 4, kRaw = 3;
    static constexpr int kRawSlot = Geo<D, 1>::kTile + 256; // a tile, and the stage's scales
    static constexpr int kArea = FP8 && kRaw * kRawSlot > kPfStageBytes ? kRaw * kRawSlot : kPfStageBytes;
    static constexpr int kAreas = kSlots * Geo<D, 2>::kStage; // the areas follow the ring
    static constexpr int kBytes = kAreas + kArea * kExWaves;
};

template <int D, bool FP8> __global__ __launch_bounds__(64 * kExWaves, D == 64 ? 3 : 2) void extend_tile_kernel(EX_PARAMS)
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

    ex_walk<kExTileRows>(a, lds, [&](const ExPlace &p, const ExPart &t) __attribute__((always_inline)) {
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
            sc_put = {scale(w[0], true) * a.scale_log2, scale(w[2], true) * a.scale_log2, scale(w[1], false), scale(w[3], false)};
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
#pragma unroll 1
                for (; s + 1 < free; s++) {
                    open(s + 1);
                    EX_STEP(false, true);
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
            float *const o = a.part_o + (int64_t)t.slot * (kExTileRows * D) + wave * (kPfRows * D) + 4 * lane;
#pragma unroll
            for (int dt = 0; dt < D / 32; dt++) {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (exists) *(f32x4 *)(o + 256 * (4 * dt + j)) = f32x4{st.o[dt][4 * j], st.o[dt][4 * j + 1], st.o[dt][4 * j + 2], st.o[dt][4 * j + 3]};
            }
            if (exists && hh == 0) *(float2 *)(a.part_lse + 2 * ((int64_t)t.slot * kExTileRows + kPfRows * wave + n)) = make_float2(st.m, l);
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
    });
    wait_vmcnt<0>(); // nothing may land in LDS after the workgroup has left
}

// ---- few rows -------------------------------------------------------------------------------------------

template <int D, int KVB> struct ExFewLds {
    using G = Geo<D, KVB>;
    static constexpr int kSlots = KVB == 2 ? 2 : 4;        // a wave's ring, in stages
    static constexpr int kRing = kSlots * G::kStage;
    static constexpr int kStats = kExWaves * kRing;         // what the waves' rows have as maximum and sum
    static constexpr int kBytes = kStats + kExWaves * kExFewRows * 8;
    static_assert(kRing >= kExFewRows * D * 4, "a wave's sums take the place of its ring");
    static_assert((kSlots - 1) * G::kDmaPerStage < 64, "the vector-memory counter holds 6 bits");
};

// NQT: tiles of sixteen rows that a sequence and kv head has at most.
template <int D, int KVB, int NQT> __global__ __launch_bounds__(64 * kExWaves, 1) void extend_few_kernel(EX_PARAMS)
{
    EX_TAKE(a);
    using G = Geo<D, KVB>;
    using X = ExFewLds<D, KVB>;
    constexpr int NST = X::kSlots, DPS = G::kDmaPerStage, W = kExWaves;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int rn = lane & 15, j = lane >> 4;
    uint8_t *const ring = lds + wave * X::kRing;
    const uint32_t ring_addr = (uint32_t)(uintptr_t)ring;
    LaneConst<D, KVB> lc;
    lane_setup<D, KVB>(lc, lane, a.stride_token_b);

    ex_walk<kExFewRows>(a, lds, [&](const ExPlace &p, const ExPart &t) __attribute__((always_inline)) {
        const int ntiles = (t.rows + 15) >> 4, shift = p.s.L - p.s.n;
        // the wave's stages of the part: wave, wave + 4, ...
        const int left = t.hi - t.lo - wave, mine = left > 0 ? (left + W - 1) / W : 0;
        const int32_t *const pages = a.table + (int64_t)p.b * a.max_pages;
        const int count = (p.s.L + kPage - 1) / kPage;
        const int64_t head_b = (int64_t)t.kvh * a.stride_head_b;
        const int last_page = count > 0 ? count - 1 : 0; // (a page that does not exist takes its place, and none of its rows are read)
        auto page_id = [&](int i, int h) __attribute__((always_inline)) {
            const int g = 2 * (t.lo + wave + W * i) + h;
            return uniform_load(pages, g < last_page ? g : last_page);
        };
        int issued = 0, id0 = 0, id1 = 0;
        if (mine > 0) id0 = page_id(0, 0), id1 = page_id(0, 1);
        auto issue = [&]() __attribute__((always_inline)) {
            if (issued >= mine) return;
            const int nv0 = p.s.L - 2 * kPage * (t.lo + wave + W * issued), nv1 = nv0 - kPage;
            const int64_t off0 = (int64_t)id0 * a.stride_page_b + head_b, off1 = (int64_t)id1 * a.stride_page_b + head_b;
            const uint32_t sb = ring_addr + (issued % NST) * G::kStage;
            issue_tile<D, KVB, true>(lc, a.k_pool + off0, nv0, sb, a.zeros);
            issue_tile<D, KVB, true>(lc, a.k_pool + off1, nv1, sb + G::kTile, a.zeros);
            issue_tile<D, KVB, true>(lc, a.v_pool + off0, nv0, sb + 2 * G::kTile, a.zeros);
            issue_tile<D, KVB, true>(lc, a.v_pool + off1, nv1, sb + 3 * G::kTile, a.zeros);
            if (KVB == 1) { // the pages' scales land behind the tiles: lanes 0..3 bring k0, v0, k1, v1
                const int pid = (lane & 2) ? id1 : id0;
                const void *src = a.zeros;
                if (lane < 4 && ((lane & 2) ? nv1 : nv0) > 0) src = ((lane & 1) ? a.v_scale : a.k_scale) + (int64_t)pid * a.Hkv + t.kvh;
                dma4(src, sb + 4 * G::kTile);
            }
            issued++;
            id0 = page_id(issued, 0), id1 = page_id(issued, 1);
        };
        // Query rows as the second operand of K . Q^T wants them: lane (row, j) holds the d values that its K operand holds.
        bf16x8 qf[NQT][G::kKSteps];
        int lim[NQT];
#pragma unroll
        for (int q = 0; q < NQT; q++) {
            int r = 16 * q + rn;
            r = r < t.rows ? r : t.rows - 1;
            const int token = ex_div_g(a, r);
            lim[q] = shift + token;
            const uint16_t *const src = a.q + (int64_t)(p.s.t0 + token) * a.q_stride + (t.kvh * a.G + r - token * a.G) * D;
#pragma unroll
            for (int i = 0; i < G::kKSteps; i++) {
                const int d0 = KVB == 2 ? 32 * i + 8 * j : 16 * (4 * (i / 2) + j) + 8 * (i % 2);
                if (q < ntiles) qf[q][i] = *(const bf16x8 *)(src + d0);
            }
        }
#pragma unroll
        for (int i = 0; i < NST - 1; i++) issue();

        f32x4 o[NQT][G::kDTiles];
        float m[NQT], lsum[NQT];
#pragma unroll
        for (int q = 0; q < NQT; q++) {
            m[q] = kPfLowest, lsum[q] = 0.f;
#pragma unroll
            for (int dt = 0; dt < G::kDTiles; dt++) o[q][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll 1
        for (int it = 0; it < mine; it++) {
            issue();
            WaitTail<NST - 1, DPS>::run(issued - 1 - it);
            const uint8_t *const st = ring + (it % NST) * G::kStage;
            const int key = 32 * (t.lo + wave + W * it);
            f32x4 s[NQT][2];
#pragma unroll
            for (int pg = 0; pg < 2; pg++) {
#pragma unroll
                for (int q = 0; q < NQT; q++) s[q][pg] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < G::kKReads; i++) {
                    if (KVB == 2) {
                        const bf16x8 kf = *(const bf16x8 *)(st + pg * G::kTile + lc.k_off[i]);
#pragma unroll
                        for (int q = 0; q < NQT; q++)
                            if (q < ntiles) s[q][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[q][i], s[q][pg], 0, 0, 0);
                    } else {
                        const int4 kc = *(const int4 *)(st + pg * G::kTile + lc.k_off[i]); // 16 codes: two k-steps
                        const bf16x8 k0 = fp8x8_to_bf16(kc.x, kc.y), k1 = fp8x8_to_bf16(kc.z, kc.w);
#pragma unroll
                        for (int q = 0; q < NQT; q++)
                            if (q < ntiles) {
                                s[q][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[q][2 * i], s[q][pg], 0, 0, 0);
                                s[q][pg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[q][2 * i + 1], s[q][pg], 0, 0, 0);
                            }
                    }
                }
            }
            // e4m3: the K scale folds into the score's, the V scale into the weights before they are rounded to bf16 (the
            // row sum keeps them unscaled)
            float ks0 = a.scale_log2, ks1 = a.scale_log2, vs0 = 1.0f, vs1 = 1.0f;
            if (KVB == 1) {
                const f32x4 sc = *(const f32x4 *)(st + 4 * G::kTile);
                ks0 *= sc[0], vs0 = sc[1], ks1 *= sc[2], vs1 = sc[3];
            }
            const bool masked = key + 31 > shift; // (the first row sees the least)
            bf16x8 pf[NQT];
#pragma unroll
            for (int q = 0; q < NQT; q++) {
                if (q >= ntiles) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = s[q][0][e] * ks0, v[4 + e] = s[q][1][e] * ks1;
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        if (key + 4 * j + e > lim[q]) v[e] = -INFINITY;
                        if (key + kPage + 4 * j + e > lim[q]) v[4 + e] = -INFINITY;
                    }
                }
                const float mx = row_max3(max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], v[7])));
                const float mn = max3(m[q], mx, mx);
                f32x8 w;
#pragma unroll
                for (int e = 0; e < 8; e++) w[e] = __builtin_amdgcn_exp2f(v[e] - mn);
                const float ws = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
                if (KVB == 1) {
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] *= vs0, w[4 + e] *= vs1;
                }
                pf[q] = __builtin_convertvector(w, bf16x8);
                if (__any(mn != m[q])) {
                    const float alpha = __builtin_amdgcn_exp2f(m[q] - mn);
                    m[q] = mn;
                    lsum[q] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < G::kDTiles; dt++) o[q][dt] *= alpha;
                }
                lsum[q] += ws;
            }
            typedef s16x4 __attribute__((address_space(3))) * lds_s16x4;
            typedef int __attribute__((ext_vector_type(2))) i32x2;
            typedef i32x2 __attribute__((address_space(3))) * lds_i32x2;
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            const uint32_t vb = ring_addr + (it % NST) * G::kStage + 2 * G::kTile;
#pragma unroll
            for (int dt = 0; dt < G::kDTiles; dt++) {
                bf16x8 vf;
                if (KVB == 2) {
                    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb + lc.v_off[dt]));
                    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(vb + G::kTile + lc.v_off[dt]));
                    vf = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    const i32x2 vc = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)((vb + lc.v_off[0]) ^ (uint32_t)(16 * dt)));
                    vf = fp8x8_to_bf16(vc[0], vc[1]);
                }
                if (masked && __builtin_expect(__any(ex_odd(vf)), 0)) {
#pragma unroll 1
                    for (int i = 0; i < 32; i++) { // element e of lane group h: key 4 h + e of the first page, or 4 h + e - 4 of the second
                        const int e = i & 7, h = i >> 3, at = key + 4 * h + (e & 3) + (e & 4 ? kPage : 0);
                        const bf16x8 one = ex_only(vf, j == h, e);
#pragma unroll
                        for (int q = 0; q < NQT; q++) {
                            if (q >= ntiles) continue;
                            const f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, pf[q], (f32x4{0.f, 0.f, 0.f, 0.f}), 0, 0, 0);
#pragma unroll
                            for (int c = 0; c < 4; c++) o[q][dt][c] += at <= lim[q] ? x[c] : 0.f;
                        }
                    }
                    continue;
                }
#pragma unroll
                for (int q = 0; q < NQT; q++)
                    if (q < ntiles) o[q][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[q], o[q][dt], 0, 0, 0);
            }
            // every LDS read of this stage has returned before a later load may overwrite it
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }

        // The four waves' sums: a row's 16-byte pieces lie XOR-swizzled by the row, in the wave's ring.
        float *const mine_o = (float *)ring;
        float2 *const stats = (float2 *)(lds + X::kStats);
        constexpr int PIECES = D / 4;
#pragma unroll
        for (int q = 0; q < NQT; q++) {
            if (q >= ntiles) continue;
            const int r = 16 * q + rn;
            const float l = row_sum(lsum[q]);
#pragma unroll
            for (int dt = 0; dt < G::kDTiles; dt++) *(f32x4 *)(mine_o + r * D + 4 * ((4 * dt + j) ^ rn)) = o[q][dt];
            if (j == 0) stats[wave * kExFewRows + r] = make_float2(m[q], l);
        }
        __syncthreads();
        for (int x = threadIdx.x; x < t.rows * PIECES; x += 64 * W) {
            const int r = x / PIECES, c = x % PIECES;
            float mm = kPfLowest, l = 0.f;
            float2 ml[W];
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < W; w++) ml[w] = stats[w * kExFewRows + r], mm = fmaxf(mm, ml[w].x);
#pragma unroll
            for (int w = 0; w < W; w++) {
                const float f = __builtin_amdgcn_exp2f(ml[w].x - mm);
                l += f * ml[w].y;
                acc += f * *(const f32x4 *)((const float *)(lds + w * X::kRing) + r * D + 4 * (c ^ (r & 15)));
            }
            if (t.slot >= 0) {
                *(f32x4 *)(a.part_o + ((int64_t)t.slot * kExFewRows + r) * D + 4 * c) = acc;
                if (c == 0) *(float2 *)(a.part_lse + 2 * ((int64_t)t.slot * kExFewRows + r)) = make_float2(mm, l);
            } else {
                const int token = ex_div_g(a, r);
                const int64_t rh = (int64_t)(p.s.t0 + token) * a.Hq + t.kvh * a.G + (r - token * a.G);
                const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l; // (no key: zeros; NaN stays)
                *(bf16x4 *)(a.out + rh * D + 4 * c) = __builtin_convertvector(acc * inv, bf16x4);
                if (c == 0) a.lse[rh] = (mm + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
            }
        }
        __syncthreads(); // (the rings take the next part's stages)
    });
    wait_vmcnt<0>();
}

// ---- what spans share -----------------------------------------------------------------------------------

constexpr int kExMergeWgs = 2048, kExMaxSpans = 1024;
constexpr int kExMergeFew = 12; // parts of an item that one wave adds up

// Adds up the parts of the items that a cut goes through, 256 consecutive values of an item's parts at a time: a wave alone
// where every item has few parts, else a workgroup's waves every fourth part each.  ROWS: those of the kernel that left them,
// with its layout.
template <int D, int ROWS> __global__ __launch_bounds__(64 * kExWaves) void extend_merge_kernel(const int4 *__restrict__ desc, int spans, ExtendLaunch given)
{
    ExtendLaunch a = given;
    a.desc = (int4 *)desc, a.spans = spans;
    touch_lines(given);
    constexpr int W = kExWaves, CHUNKS = ROWS * D / 256, N = kExMaxSpans / (64 * W);
    __shared__ int list[kExMaxSpans];
    __shared__ int counts[W][N], longest[W];
    __shared__ f32x4 sums[W][64];
    __shared__ float2 stats[W][64];
    const int lane = threadIdx.x & 63, wave = ex_uni((int)threadIdx.x >> 6);
    // the spans in which such an item begins, in order
    int ends[N], most = 0, items = 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int k = 64 * W * i + (int)threadIdx.x;
        ends[i] = k < a.spans ? a.desc[2 * k + 1].x : 0;
    }
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int k = 64 * W * i + (int)threadIdx.x;
        most = most > ends[i] - k ? most : ends[i] - k;
        const int n = __popcll(__ballot(ends[i] > k));
        if (lane == 0) counts[wave][i] = n;
    }
    const bool long_ones = __any(most >= kExMergeFew);
    if (lane == 0) longest[wave] = long_ones;
    __syncthreads();
    bool split = false;
#pragma unroll
    for (int w = 0; w < W; w++) split = split || longest[w];
#pragma unroll
    for (int i = 0; i < N; i++) {
        const int k = 64 * W * i + (int)threadIdx.x;
        int at = items;
#pragma unroll
        for (int w = 0; w < W; w++) {
            if (w < wave) at += counts[w][i];
            items += counts[w][i];
        }
        const unsigned long long m = __ballot(ends[i] > k);
        if (ends[i] > k) list[at + __popcll(m & ((1ull << lane) - 1ull))] = k;
    }
    __syncthreads();
    const int each = split ? 1 : W; // units of work that a workgroup takes at a time
    for (int u0 = blockIdx.x * each; u0 < items * CHUNKS; u0 += gridDim.x * each) {
        const int u = split ? u0 : u0 + wave, chunk = u % CHUNKS;
        const bool have = u < items * CHUNKS;
        const int k = list[have ? u / CHUNKS : 0];
        const int4 item = a.desc[2 * k]; // {first packed token, first row, rows, kv head}
        const int last = a.desc[2 * k + 1].x;
        int r, d; // this lane's row of the block, and the first of its four values
        if (ROWS == kExTileRows) {
            const int wv = chunk / (D / 8), c = chunk % (D / 8);
            r = kPfRows * wv + (lane & 31), d = 32 * (c >> 2) + 8 * (c & 3) + 4 * (lane >> 5);
        } else {
            r = chunk * (256 / D) + lane / (D / 4), d = 4 * (lane % (D / 4));
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
                        ml[i] = *(const float2 *)(a.part_lse + 2 * (slot * ROWS + r));
                        o[i] = *(const f32x4 *)(a.part_o + slot * (ROWS * D) + 256 * chunk + 4 * lane);
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
