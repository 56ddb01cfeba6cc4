// gfx950 kernels of the norm and rotation of query and key rows by head, and of the append of chunks of new tokens to the
// paged cache with both on the way.
//
// Memory bounds them: a row of D bf16 is read once and written once, and everything between stays in binary32 registers.  A
// row belongs to D / 16 lanes, each with two 16-byte units of it, chosen so that the two values that a rotation turns are in
// one lane: units j and j + rot / 16 where a pair is half the rotated part apart, neighbours where it is a pair of
// neighbours.  The only step across lanes is the sum of squares, over a row's eight or four.
//
// Measured: 16 384 tokens of 28 + 4 heads, D = 128, 53.3 us, 5.0 TB/s read and written (a copy of 1 GiB: 5.1); 7 201 of 32 + 2 heads, D =
// 64, ragged, 12.8 us; a handful 4.4 us, which is the launch and three trips.  Into pages: 8 192 tokens of 64 + 8 + 8 heads 69.3 us,
// 4.9 TB/s; one token for each of 256 sequences 4.3 us, into e4m3 pages 8.0; 6 424 tokens of 40 + 8 + 8 heads into those 44 us, 4.0 TB/s.
#include "ra_chunk.h"
#include "ra_device.h"

namespace ra {

constexpr int kRowWaves = 4;

// This lane's sixteen values of a row: the units that they are in (of eight values), and the values.
template <int D> struct RowLane {
    static constexpr int kLanes = D / 16;
    int ua, ub;
    __device__ __forceinline__ void place(int lane, int rot, int interleaved)
    {
        const int j = lane & (kLanes - 1);
        const bool near = interleaved || j >= rot / 16;
        ua = near ? 2 * j : j;
        ub = near ? 2 * j + 1 : j + rot / 16;
    }
};

struct Row {
    float x[16];
};

__device__ __forceinline__ void unpack(Row &r, uint4 a, uint4 b)
{
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; i++) r.x[2 * i] = bf16_lo(w[i]), r.x[2 * i + 1] = bf16_hi(w[i]);
}
__device__ __forceinline__ bf16x8 pack(const float *x)
{
    typedef float f32x8v __attribute__((ext_vector_type(8)));
    return __builtin_convertvector((f32x8v{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}), bf16x8);
}

// x * w / sqrt(mean(x^2) + eps): the sum of squares over the row's lanes by exchanges inside groups of eight (or four).
template <int D> __device__ __forceinline__ void normalise(Row &r, const float (&w)[16], float eps)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i++) s = __builtin_fmaf(r.x[i], r.x[i], s);
#pragma unroll
    for (int sh = 1; sh < RowLane<D>::kLanes; sh *= 2) s += __shfl_xor(s, sh);
    const float inv = rsqrtf(s * (1.0f / D) + eps);
#pragma unroll
    for (int i = 0; i < 16; i++) r.x[i] = r.x[i] * inv * w[i];
}

// Cosines and sines of this lane's eight pairs: pair i is (x[i], x[8 + i]), or with neighbours (x[2 i], x[2 i + 1]).
struct Turn {
    float c[8], s[8];
};
template <int D> __device__ __forceinline__ void load_turn(Turn &t, const RowsLaunch &a, const RowLane<D> &rl, int lane, int position)
{
    const float *const row = a.rope + (int64_t)position * a.rot;
    const int half = a.rot / 2, j = lane & (RowLane<D>::kLanes - 1);
    // the angles of unit ua's first pairs and of unit ub's: eight in a row, or four for each unit of neighbours
    int at0 = 8 * j, at1 = 8 * j + 4;
    bool in0 = j < a.rot / 16, in1 = in0;
    if (a.interleaved) at0 = 4 * rl.ua, at1 = 4 * rl.ub, in0 = rl.ua < a.rot / 8, in1 = rl.ub < a.rot / 8;
#pragma unroll
    for (int h = 0; h < 2; h++) {
        f32x4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
        if (h ? in1 : in0) {
            c = *(const f32x4 *)(row + (h ? at1 : at0));
            s = *(const f32x4 *)(row + half + (h ? at1 : at0));
        }
#pragma unroll
        for (int i = 0; i < 4; i++) t.c[4 * h + i] = c[i], t.s[4 * h + i] = s[i];
    }
}
// (A lane's units are rotated together or not at all: rot is a multiple of sixteen.  A lane that is not keeps its bits: no
// product with a cosine of one, which would not keep a NaN's.)
__device__ __forceinline__ void rotate(Row &r, const Turn &t, int interleaved)
{
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float x = r.x[2 * i], y = r.x[2 * i + 1];
            r.x[2 * i] = x * t.c[i] - y * t.s[i];
            r.x[2 * i + 1] = y * t.c[i] + x * t.s[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float x = r.x[i], y = r.x[8 + i];
            r.x[i] = x * t.c[i] - y * t.s[i];
            r.x[8 + i] = y * t.c[i] + x * t.s[i];
        }
    }
}

template <int D> __device__ __forceinline__ void load_weight(float (&w)[16], const float *at, const RowLane<D> &rl)
{
#pragma unroll
    for (int h = 0; h < 4; h++) {
        const f32x4 x = *(const f32x4 *)(at + 8 * (h < 2 ? rl.ua : rl.ub) + 4 * (h & 1));
#pragma unroll
        for (int i = 0; i < 4; i++) w[4 * h + i] = x[i];
    }
}

// The sequence that packed token t belongs to: the number of chunks that end at or before it.  t is the wave's.
__device__ __forceinline__ int sequence_of(const RowsLaunch &a, int t, int lane)
{
    int b = 0;
    for (int base = 0; base < a.B; base += 256) {
        int end[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int s = base + 64 * i + lane;
            end[i] = s < a.B ? a.cu[s + 1] : INT32_MAX;
        }
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) n += __popcll(__ballot(end[i] <= t));
        b += n;
        if (n < 256) break;
    }
    return b;
}

// Rows of N passes of a wave: each pass has 64 / (D / 16) row slots, 2^slots_shift of them for a token; a token with more rows
// (query heads, key heads, into a cache value heads too) than that takes the slots of several passes.
enum RowsTo { kToRows, kToPages, kBesidePages }; // rows; keys and values into pages of bf16; queries whose keys others write
template <int D, RowsTo TO, int N> __device__ __forceinline__ void rows_of_wave(const RowsLaunch &a, int unit, int lane)
{
    constexpr bool CACHE = TO == kToPages, SEQ = TO != kToRows; // tokens belong to sequences
    using R = RowLane<D>;
    constexpr int SLOTS = 64 / R::kLanes;
    const int rows = TO == kBesidePages ? a.Hq : a.Hq + a.Hkv + (CACHE ? a.Hkv : 0);
    const int per = 1 << a.slots_shift, tokens = SLOTS >> a.slots_shift; // row slots of a token, tokens of a pass
    const int groups = (rows + N * per - 1) / (N * per);                 // waves that share a token's rows (1 where tokens > 1)
    const int first = unit / groups * tokens, pass0 = (unit - unit / groups * groups) * N;
    if (first >= a.T) return;
    const int slot = lane / R::kLanes, t = first + (slot >> a.slots_shift);
    R rl;
    rl.place(lane, a.rot, a.interleaved);
    const bool live = t < a.T;
    // the rows' values are asked for before anything that has to be looked up
    int head[N];
    uint4 wa[N], wb[N];
#pragma unroll
    for (int n = 0; n < N; n++) {
        int h = (pass0 + n) * per + (slot & (per - 1));
        if (!live || h >= rows) h = -1;
        head[n] = h;
        const uint16_t *at = nullptr;
        if (h >= 0)
            at = h < a.Hq ? a.q + (int64_t)t * a.q_stride + h * D
                          : h < a.Hq + a.Hkv ? a.k + (int64_t)t * a.k_stride + (h - a.Hq) * D : a.v + (int64_t)t * a.v_stride + (h - a.Hq - a.Hkv) * D;
        if (at) wa[n] = *(const uint4 *)(at + 8 * rl.ua), wb[n] = *(const uint4 *)(at + 8 * rl.ub);
    }
    int position = -1, b = 0, at_seq = 0; // rotation, sequence, place in the sequence's cache
    uint8_t *page_k = nullptr, *page_v = nullptr;
    if (SEQ) {
        b = sequence_of(a, first, lane);
        if (live) {
            while (b < a.B && a.cu[b + 1] <= t) b++; // (a pass with several tokens: its later ones)
        }
        if (live && b < a.B) {
            const int i = t - a.cu[b];
            const int len = a.seq_lens[b];
            at_seq = (int)((unsigned)len + (unsigned)i); // (beyond 2^31 - 1: negative, no position)
            position = at_seq;
            if (CACHE && i >= 0 && i < a.max_chunk && len >= 0 && at_seq >= 0 && at_seq < a.max_pages * kPage) {
                const int pid = a.table[(int64_t)b * a.max_pages + at_seq / kPage];
                if (pid >= 0 && pid < a.num_pages) {
                    const int64_t off = (int64_t)pid * a.stride_page_b + (int64_t)(at_seq % kPage) * a.stride_token_b;
                    page_k = a.k_pool + off, page_v = a.v_pool + off;
                }
            }
        }
    }
    if (a.positions && live) position = a.positions[t];
    const bool turned = a.rot > 0;
    if (!live || (turned && (position < 0 || position >= a.rope_len)) || (SEQ && b >= a.B)) return;
    Turn turn;
    if (turned) load_turn<D>(turn, a, rl, lane, position);
    const int j = lane & (R::kLanes - 1);
    const bool mine = turned && (a.interleaved ? rl.ua < a.rot / 8 : j < a.rot / 16);
#pragma unroll
    for (int n = 0; n < N; n++) {
        const int h = head[n];
        if (h < 0) continue;
        const bool is_q = h < a.Hq, is_v = CACHE && h >= a.Hq + a.Hkv;
        uint16_t *dst;
        if (is_q) dst = a.q_out + (int64_t)t * a.q_out_stride + h * D;
        else if (!CACHE) dst = a.k_out + (int64_t)t * a.k_out_stride + (h - a.Hq) * D;
        else if (!is_v) dst = page_k ? (uint16_t *)(page_k + (h - a.Hq) * a.stride_head_b) : nullptr;
        else dst = page_v ? (uint16_t *)(page_v + (h - a.Hq - a.Hkv) * a.stride_head_b) : nullptr;
        if (!dst) continue;
        if (is_v) {
            *(uint4 *)(dst + 8 * rl.ua) = wa[n], *(uint4 *)(dst + 8 * rl.ub) = wb[n];
            continue;
        }
        Row r;
        unpack(r, wa[n], wb[n]);
        const float *const weight = is_q ? a.qw : a.kw;
        if (weight) {
            float w[16];
            load_weight<D>(w, weight, rl);
            normalise<D>(r, w, a.eps);
        }
        if (mine) rotate(r, turn, a.interleaved);
        *(bf16x8 *)(dst + 8 * rl.ua) = pack(r.x), *(bf16x8 *)(dst + 8 * rl.ub) = pack(r.x + 8);
    }
}

template <int D, RowsTo TO, int N> __global__ __launch_bounds__(64 * kRowWaves) void rows_kernel(const uint16_t *__restrict__ q, const uint16_t *__restrict__ k, int64_t q_stride, int64_t k_stride, int T,
                                                                                    int Hq, int Hkv, int slots_shift, RowsLaunch given)
{
    RowsLaunch a = given; // (what the first loads need is in registers when a wave starts)
    a.q = q, a.k = k, a.q_stride = q_stride, a.k_stride = k_stride, a.T = T, a.Hq = Hq, a.Hkv = Hkv, a.slots_shift = slots_shift;
    touch_lines(given);
    rows_of_wave<D, TO, N>(a, blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), threadIdx.x & 63);
}

// Waves that N passes each take for all rows, and the row slots of a token.
template <int D> static int64_t rows_units(RowsLaunch &a, int rows, int n)
{
    constexpr int SLOTS = 64 / RowLane<D>::kLanes;
    int shift = 0;
    while ((1 << shift) < rows && (1 << shift) < SLOTS) shift++;
    a.slots_shift = shift;
    const int per = 1 << shift, tokens = SLOTS >> shift;
    return ((int64_t)a.T + tokens - 1) / tokens * ((rows + n * per - 1) / (n * per));
}

template <int D, RowsTo TO> static hipError_t launch_rows(RowsLaunch &a, int num_cus, hipStream_t s)
{
    const int rows = a.Hq + a.Hkv + (TO == kToPages ? a.Hkv : 0);
    if (a.T == 0 || rows == 0) return hipSuccess;
    // Few rows: as many waves as there are, a pass each.  Many, into a cache: four passes, which look for their place in it once
    // (8 192 tokens of 64 + 8 + 8 heads: 75.4 -> 71.1 us; 256 tokens of 28 + 4 + 4: 4.5, with four passes 6.2).  Without a place to
    // look for a pass each is the faster also there (7 201 rotated tokens of 34 heads, D = 64: 12.6 us, with four 14.9).
    int64_t units = rows_units<D>(a, rows, 1);
    const bool many = TO != kToRows && units > 32 * (int64_t)num_cus;
    if (many) units = rows_units<D>(a, rows, 4);
    const int64_t groups = (units + kRowWaves - 1) / kRowWaves;
    if (groups > INT32_MAX) return hipErrorInvalidValue;
#define RA_ROWS(a) a.q, a.k, a.q_stride, a.k_stride, a.T, a.Hq, a.Hkv, a.slots_shift, a
    if constexpr (TO != kToRows) {
        if (many) {
            hipLaunchKernelGGL((rows_kernel<D, TO, 4>), dim3((unsigned)groups), dim3(64 * kRowWaves), 0, s, RA_ROWS(a));
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((rows_kernel<D, TO, 1>), dim3((unsigned)groups), dim3(64 * kRowWaves), 0, s, RA_ROWS(a));
#undef RA_ROWS
    return hipGetLastError();
}

hipError_t launch_rotate(const RowsLaunch &given, int num_cus, hipStream_t s)
{
    RowsLaunch a = given;
    return a.D == 128 ? launch_rows<128, kToRows>(a, num_cus, s) : launch_rows<64, kToRows>(a, num_cus, s);
}

// ------------------------------------------------------------------------------------------------------
// e4m3 pools: a wave per (page that a chunk touches, kv head) and tensor, which has the page's new rows in registers, finds
// their largest magnitude, decides on the scale and writes codes; queries are rows as above, by other waves of the launch.
// (Four passes a wave for them as for bf16 pools: 6 424 tokens of 40 heads 49.4 -> 44.0 us.  What is left to a copy's rate, 34, is
// the pages' chain of trips, sequence, page, rows, scale, with little on the way in each.)
//
// The pages are numbered without counting them: sequence b's are given the numbers from cu[b] / 16 + 2 b on, which leaves it
// n / 16 + 2 of them at least, and n new tokens touch (n + 30) / 16 pages at most.
// ------------------------------------------------------------------------------------------------------

__device__ __forceinline__ int page_number(int cu, int b) { return (cu >> 4) + 2 * b; }

// The four stored codes of a dword from scale `old` to scale sc.s: code' = enc((dec(code) * old) / sc.s).
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float old, const E4m3Scale &sc, bool fast)
{
    if (fast && !(((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u)) // no NaN among the four
        return sc.codes4(__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * old, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * old,
                         __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * old, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * old);
    uint32_t r = 0;
#pragma unroll 1
    for (int e = 0; e < 4; e++) r |= e4m3_nearest((e4m3_value((w >> (8 * e)) & 0xff) * old) / sc.s) << (8 * e);
    return r;
}
__device__ __forceinline__ uint2 codes8(const float *x, const E4m3Scale &sc, bool fast)
{
    if (fast) return make_uint2(sc.codes4(x[0], x[1], x[2], x[3]), sc.codes4(x[4], x[5], x[6], x[7]));
    uint32_t r[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e++) r[e >> 2] |= e4m3_nearest(x[e] / sc.s) << (8 * (e & 3));
    return make_uint2(r[0], r[1]);
}

template <int D> __device__ __forceinline__ void page_of_wave(const RowsLaunch &a, int unit, int lane)
{
    using R = RowLane<D>;
    constexpr int SLOTS = 64 / R::kLanes, NR = kPage / SLOTS; // rows at a time, times
    const bool is_v = unit & 1;
    const int item = unit >> 1, number = item / a.Hkv, kvh = item - number * a.Hkv;
    // the last sequence whose numbers start at or before this one
    int b = -1;
    for (int base = 0; base < a.B; base += 256) {
        int n = 0, start[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int s = base + 64 * i + lane;
            start[i] = s < a.B ? page_number(a.cu[s], s) : INT32_MAX;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) n += __popcll(__ballot(start[i] <= number));
        b += n;
        if (n < 256) break;
    }
    if (b < 0) return;
    const int t0 = uniform_load(a.cu, b), before = uniform_load(a.seq_lens, b);
    int n = uniform_load(a.cu, b + 1) - t0;
    if (t0 < 0 || n <= 0 || n > a.T - t0) return;
    n = n < a.max_chunk ? n : a.max_chunk;
    if (before < 0 || before >= a.max_pages * kPage) return;
    const int page = before / kPage + (number - page_number(t0, b)); // in the sequence's table
    const int64_t end = (int64_t)before + n;
    if (page >= a.max_pages || (int64_t)page * kPage >= end) return;
    const int lo = page * kPage > before ? 0 : before - page * kPage; // the new rows' slots
    const int hi = end - (int64_t)page * kPage < kPage ? (int)(end - (int64_t)page * kPage) : kPage;
    const int pid = uniform_load(a.table, (int64_t)b * a.max_pages + page);
    if (pid < 0 || pid >= a.num_pages) return;
    R rl;
    rl.place(lane, is_v ? 0 : a.rot, a.interleaved);
    Row r[NR];
    bool in[NR];
    const int slot0 = lane / R::kLanes;
    const int64_t stride = is_v ? a.v_stride : a.k_stride;
    const uint16_t *const src = (is_v ? a.v : a.k) + (int64_t)kvh * D;
    const float *const weight = is_v ? nullptr : a.kw;
    const bool turned = !is_v && a.rot > 0;
    uint4 wa[NR], wb[NR];
#pragma unroll
    for (int i = 0; i < NR; i++) {
        const int slot = SLOTS * i + slot0;
        in[i] = slot >= lo && slot < hi;
        wa[i] = wb[i] = make_uint4(0, 0, 0, 0);
        if (in[i]) {
            const uint16_t *const at = src + (int64_t)(t0 + (page * kPage + slot - before)) * stride;
            wa[i] = *(const uint4 *)(at + 8 * rl.ua), wb[i] = *(const uint4 *)(at + 8 * rl.ub);
        }
    }
    uint8_t *const tile = (is_v ? a.v_pool : a.k_pool) + (int64_t)pid * a.stride_page_b + (int64_t)kvh * a.stride_head_b;
    float *const scale_ptr = (is_v ? a.v_scale : a.k_scale) + (int64_t)pid * a.Hkv + kvh;
    const float old = lo ? *scale_ptr : 0.f;
    float w[16];
    if (weight) load_weight<D>(w, weight, rl);
    float amax = 0.f;
    bool odd = false; // a NaN
    const int j = lane & (R::kLanes - 1);
    const bool mine = turned && (a.interleaved ? rl.ua < a.rot / 8 : j < a.rot / 16);
#pragma unroll
    for (int i = 0; i < NR; i++) {
        const int place = page * kPage + SLOTS * i + slot0;
        unpack(r[i], wa[i], wb[i]);
        int position = place;
        if (a.positions && in[i]) position = a.positions[t0 + (place - before)];
        // (a token that cannot be rotated is left out, its value too)
        if (a.rot > 0 && (position < 0 || position >= a.rope_len)) in[i] = false;
        if (weight) normalise<D>(r[i], w, a.eps);
        if (mine && in[i]) {
            Turn turn;
            load_turn<D>(turn, a, rl, lane, position);
            rotate(r[i], turn, a.interleaved);
        }
        if (in[i]) {
#pragma unroll
            for (int e = 0; e < 16; e++) {
                amax = fmaxf(amax, fabsf(r[i].x[e]));
                odd = odd || r[i].x[e] != r[i].x[e];
            }
        }
    }
#pragma unroll
    for (int sh = 32; sh; sh >>= 1) amax = fmaxf(amax, __shfl_xor(amax, sh));
    float s = old;
    if (lo == 0) {
        s = amax > 0.f ? amax / 448.0f : 1.0f;
    } else if (!(amax <= old * 448.0f)) {
        s = amax / 448.0f;
        const E4m3Scale sc = {s, 1.0f / s};
        const bool fast = E4m3Scale::ok(amax) && old >= 0.f; // (then old < amax / 448: no stored value exceeds 448 s)
#pragma unroll
        for (int i = 0; i < NR; i++) {
            const int slot = SLOTS * i + slot0;
            if (slot >= lo) continue;
            uint4 *const at = (uint4 *)(tile + (int64_t)slot * a.stride_token_b + 16 * j);
            const uint4 c = *at;
            *at = make_uint4(rescale4(c.x, old, sc, fast), rescale4(c.y, old, sc, fast), rescale4(c.z, old, sc, fast), rescale4(c.w, old, sc, fast));
        }
    }
    // codes by the quick quotient where it is exact: no value above the scale's range, no NaN
    const E4m3Scale sc = {s, 1.0f / s};
    const bool fast = E4m3Scale::ok(amax) && E4m3Scale::ok(448.0f * s) && !__any(odd);
#pragma unroll
    for (int i = 0; i < NR; i++) {
        if (!in[i]) continue;
        uint8_t *const at = tile + (int64_t)(SLOTS * i + slot0) * a.stride_token_b;
        *(uint2 *)(at + 8 * rl.ua) = codes8(r[i].x, sc, fast);
        *(uint2 *)(at + 8 * rl.ub) = codes8(r[i].x + 8, sc, fast);
    }
    if (lane == 0) *scale_ptr = s;
}

template <int D, int N> __global__ __launch_bounds__(64 * kRowWaves) void append_pages_kernel(const int32_t *__restrict__ cu, int B, int Hkv, int page_groups, int page_units, RowsLaunch given)
{
    RowsLaunch a = given;
    a.cu = cu, a.B = B, a.Hkv = Hkv;
    touch_lines(given);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    if ((int)blockIdx.x < page_groups) {
        const int unit = blockIdx.x * kRowWaves + wave;
        if (unit < page_units) page_of_wave<D>(a, unit, lane);
        return;
    }
    rows_of_wave<D, kBesidePages, N>(a, ((int)blockIdx.x - page_groups) * kRowWaves + wave, lane);
}

hipError_t launch_append_chunk(const RowsLaunch &given, int kv_fp8, int num_cus, hipStream_t s)
{
    RowsLaunch a = given;
    if (!kv_fp8) return a.D == 128 ? launch_rows<128, kToPages>(a, num_cus, s) : launch_rows<64, kToPages>(a, num_cus, s);
    if (a.T == 0) return hipSuccess;
    const int64_t page_units = ((int64_t)(a.T >> 4) + 2 * (int64_t)a.B) * a.Hkv * 2, page_groups = (page_units + kRowWaves - 1) / kRowWaves;
    int64_t row_units = 0;
    bool many = false;
    if (a.Hq) {
        row_units = a.D == 128 ? rows_units<128>(a, a.Hq, 1) : rows_units<64>(a, a.Hq, 1);
        many = row_units > 32 * (int64_t)num_cus;
        if (many) row_units = a.D == 128 ? rows_units<128>(a, a.Hq, 4) : rows_units<64>(a, a.Hq, 4);
    }
    const int64_t groups = page_groups + (row_units + kRowWaves - 1) / kRowWaves;
    if (groups > INT32_MAX || page_units > INT32_MAX) return hipErrorInvalidValue;
#define RA_APPEND(DD, N) \
    hipLaunchKernelGGL((append_pages_kernel<DD, N>), dim3((unsigned)groups), dim3(64 * kRowWaves), 0, s, a.cu, a.B, a.Hkv, (int)page_groups, (int)page_units, a)
    if (a.D == 128) {
        if (many) RA_APPEND(128, 4);
        else RA_APPEND(128, 1);
    } else {
        if (many) RA_APPEND(64, 4);
        else RA_APPEND(64, 1);
    }
#undef RA_APPEND
    return hipGetLastError();
}

} // namespace ra
