// gfx950 kernels of the verification of drafted tokens and the choice of next ones.
//
// p = softmax(l / T) over rows of many thousand logits, from which one token is drawn by a running sum.  The borders of that sum
// decide, and there are as many as tokens: with binary32 weights each moves by some 2^-26 of the whole, which over 150 000 of them
// changes one token in a few hundred.  So tests and draws are those of binary64 weights and sums, whose instructions this machine issues
// nearly as fast as binary32 ones; but a weight is 17 of them, against 5, and that is over the memory's pace for bf16 logits.  Where there
// are many, sums are of binary32 weights first; they come with a bound on their error (verify_shape), and what they do not settle is
// done again in binary64.
//
// A call is: the sums of the rows, in parts of 4096 values (verify_rows_kernel, verify_few_rows_kernel); tests and draws, by the parts' sums
// and one part again (verify_draw_kernel); and the draws that it leaves open, from p - q and those in doubt (verify_again_kernel,
// verify_rest_kernel, or verify_left_kernel and verify_close_kernel).
//
// Memory bounds the sums of large batches: 200 x 4 to 6 rows of 152 064 binary32 logits with a draft model's 179 us, 6.1 TB/s; 128 x 5 of
// bf16 62 to 67, 5.2 to 5.6 TB/s; binary64 sums take 22 to 24 us for 24 million values, their instructions.  The draws are chains of
// trips to memory, 6 to 10 us a kernel, and so is a small call: 4 rows of 32 000 in 9.4 us.
#include "ra_device.h"
#include "ra_step.h"
#include "ra_wave.h"

namespace ra {

constexpr int kVerifyThreads = 256;
constexpr int kDrawThreads = 512, kDrawWaves = kDrawThreads / 64;
constexpr int kVec = 8;                                          // values that a lane loads at a time
constexpr double kLog2e = 1.4426950408889634074;

// What a row's weights are made with: 2^((l - top) * c).
struct Temper {
    double c;                    // log2(e) / T; 0: greedy
    double low;                  // differences at or below this weigh nothing: 2^-1100
    float cf;
};
__device__ __forceinline__ Temper temper_from(float T)
{
    if (!(T > 0.f)) return {0.0, 0.0, 0.f};
    T = T < 1e-30f ? 1e-30f : T > 1e30f ? 1e30f : T;
    const double c = kLog2e / (double)T;
    return {c, -1100.0 / kLog2e * (double)T, (float)c};
}

// 2^x for x = d * c >= -1100, right to 2^-39: to the nearest whole number (by an addition that leaves it in the low bits), and for the
// rest the polynomial of degree eight through 2^x at nine Chebyshev nodes of [-1/2, 1/2], with the constant term at 1.
__device__ __forceinline__ double power(double d, double c)
{
    constexpr double kRound = 6755399441055744.0;               // 3 * 2^51
    const double z = __builtin_fma(d, c, kRound);
    const double f = __builtin_fma(d, c, kRound - z);
    double p = 1.3255224887502117e-06;
    p = __builtin_fma(p, f, 1.531007940254368e-05);
    p = __builtin_fma(p, f, 0.0001540345585240991);
    p = __builtin_fma(p, f, 0.0013333450567999414);
    p = __builtin_fma(p, f, 0.009618129159402628);
    p = __builtin_fma(p, f, 0.05550410941205934);
    p = __builtin_fma(p, f, 0.2402265069581299);
    p = __builtin_fma(p, f, 0.6931471805459335);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)__double_as_longlong(z));
}
// The weight of logit l against top, which is finite and not smaller by much: 0 for -inf.
__device__ __forceinline__ double weight(float l, double top, const Temper &t)
{
    return power(__builtin_fmax((double)l - top, t.low), t.c);
}

// The same in binary32, off by no more than (3 ln 2 |y| + 2) 2^-24 of it, y = (l - top) c: the difference, c and the product are rounded,
// and the instruction's own step.
__device__ __forceinline__ float weight32(float l, float top, const Temper &t) { return __builtin_amdgcn_exp2f((l - top) * t.cf); }
__device__ __forceinline__ float sum_of_eight(const float (&x)[kVec])
{
    return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}

// The larger of the two, or NaN if one is.
__device__ __forceinline__ float top_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// What a sum against `from` has to be multiplied by to stand against `to`, which is not smaller.
__device__ __forceinline__ double rescale(float from, float to, const Temper &t)
{
    return power(__builtin_fmax((double)from - (double)to, t.low), t.c);
}

__device__ __forceinline__ double last_lane(double x)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), 63), __builtin_amdgcn_readlane(__double2loint(x), 63));
}
__device__ __forceinline__ double lane_of(double x, int lane)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), lane), __builtin_amdgcn_readlane(__double2loint(x), lane));
}
__device__ __forceinline__ double wave_sum(double x) { return last_lane(wave_scan(x)); }
template <int CTRL, int ROWS> __device__ __forceinline__ float top_from_lane(float x)
{
    return top_of(x, __int_as_float(from_lane<CTRL, ROWS>(__float_as_int(x), __float_as_int(-INFINITY))));
}
__device__ __forceinline__ float wave_top(float x)
{
    x = top_from_lane<0x111, 0xf>(x);
    x = top_from_lane<0x112, 0xf>(x);
    x = top_from_lane<0x114, 0xf>(x);
    x = top_from_lane<0x118, 0xf>(x);
    x = top_from_lane<0x142, 0xa>(x);
    x = top_from_lane<0x143, 0xc>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
template <int CTRL, int ROWS> __device__ __forceinline__ int less_from_lane(int x)
{
    const int o = from_lane<CTRL, ROWS>(x, INT32_MAX);
    return o < x ? o : x;
}
__device__ __forceinline__ int wave_least(int x)
{
    x = less_from_lane<0x111, 0xf>(x);
    x = less_from_lane<0x112, 0xf>(x);
    x = less_from_lane<0x114, 0xf>(x);
    x = less_from_lane<0x118, 0xf>(x);
    x = less_from_lane<0x142, 0xa>(x);
    x = less_from_lane<0x143, 0xc>(x);
    return __builtin_amdgcn_readlane(x, 63);
}

// Sixteen bytes from anywhere an element may lie.
template <bool FP32> struct Words {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Words<false> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
};

template <bool FP32> struct Row {
    const uint8_t *at;
    static constexpr int kBytes = FP32 ? 4 : 2;
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (FP32) return ((const float *)at)[i];
        else return __uint_as_float((uint32_t)((const uint16_t *)at)[i] << 16);
    }
    // Values i .. i + 7 as they lie there (a row begins at any element: the load is of no alignment but that), and as they are.  STREAM:
    // with the hint that they are read once.
    typedef typename Words<FP32>::type words;
    struct Raw {
        words w[FP32 ? 2 : 1];
    };
    template <bool STREAM = false> __device__ __forceinline__ Raw ask(int i) const
    {
        const words *const from = (const words *)(at + (size_t)i * kBytes);
        Raw r;
#pragma unroll
        for (int j = 0; j < (FP32 ? 2 : 1); j++) r.w[j] = STREAM ? __builtin_nontemporal_load(from + j) : from[j];
        return r;
    }
    static __device__ __forceinline__ void take(float (&x)[kVec], const Raw &r)
    {
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if constexpr (FP32) x[j] = __uint_as_float(r.w[0][j]), x[4 + j] = __uint_as_float(r.w[1][j]);
            else x[2 * j] = __uint_as_float(r.w[0][j] << 16), x[2 * j + 1] = __uint_as_float(r.w[0][j] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void load(float (&x)[kVec], int i) const { take(x, ask(i)); }
    // ... of which those at or past end are -inf.
    __device__ __forceinline__ void load_some(float (&x)[kVec], int i, int end) const
    {
        if (i + kVec <= end) { load(x, i); return; }
#pragma unroll
        for (int j = 0; j < kVec; j++) x[j] = i + j < end ? (*this)[i + j] : -INFINITY;
    }
};

__device__ __forceinline__ bool is_finite(float x) { return __builtin_isfinite(x); }

// ---- a part of a row ----------------------------------------------------------------------------------

// What a thread knows of the values that it has met: the largest, their weights' sum against `mine`, and for a greedy row the first of the
// largest.  `mine` is a value that it met, and moves to a larger one only where weights would grow past 2^500 (in binary32: 2^8).
template <bool EXACT> struct Met {
    float top = -INFINITY, mine = -__FLT_MAX__;
    int first = INT32_MAX;
    double sum = 0.0, against = -__FLT_MAX__;
    __device__ __forceinline__ void meet(float (&x)[kVec], int i, const Temper &t, bool greedy)
    {
        float m = x[0];
#pragma unroll
        for (int j = 1; j < kVec; j++) m = top_of(m, x[j]);
        if (greedy) {
            if (m > top)
#pragma unroll
                for (int j = kVec - 1; j >= 0; j--)
                    if (x[j] == m) first = i + j;
        } else {
            if ((m - mine) * t.cf > (EXACT ? 500.f : 8.f)) {    // (also the first time)
                sum *= rescale(mine, m, t);
                mine = m, against = m;
            }
            if constexpr (EXACT) {
#pragma unroll
                for (int j = 0; j < kVec; j++) sum += weight(x[j], against, t);
            } else {
#pragma unroll
                for (int j = 0; j < kVec; j++) x[j] = weight32(x[j], mine, t);
                sum += (double)sum_of_eight(x);
            }
        }
        top = top_of(top, m);
    }
};

// Values [begin, end) of a row, by THREADS threads of which this is number tid: two loads of eight values are on their way at a time (the rows'
// sums of 128 x 5 bf16 rows of 152 064 values and a draft model's 62 us; with four 69, with one 2 to 4 % more), then one, then what is left
// of a load, a value to a thread.
template <bool EXACT, int THREADS, bool FP32> __device__ __forceinline__ Met<EXACT> meet_all(const Row<FP32> row, int begin, int end, const Temper &t, int tid)
{
    constexpr int kAhead = 2, kStep = THREADS * kVec;
    const bool greedy = t.c == 0.0;
    const int whole = begin + ((end - begin) & ~(kVec - 1));
    Met<EXACT> met;
    float x[kVec];
    int i = begin + tid * kVec;
    for (; i + (kAhead - 1) * kStep < whole; i += kAhead * kStep) {
        typename Row<FP32>::Raw r[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; j++) r[j] = row.template ask<!EXACT>(i + j * kStep);
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            row.take(x, r[j]);
            met.meet(x, i + j * kStep, t, greedy);
        }
    }
    for (; i < whole; i += kStep) {
        row.load(x, i);
        met.meet(x, i, t, greedy);
    }
    if (whole + tid < end) {
        x[0] = row[whole + tid];
#pragma unroll
        for (int j = 1; j < kVec; j++) x[j] = -INFINITY;
        met.meet(x, whole + tid, t, greedy);
    }
    return met;
}

// The lanes of a wave together: `all` is the largest over whatever the sum is to stand against.
template <bool EXACT> __device__ __forceinline__ RowPart wave_part(const Met<EXACT> &met, float all, const Temper &t)
{
    RowPart r = {0.0, all, INT32_MAX};
    if (t.c == 0.0) r.first = wave_least(met.top == all ? met.first : INT32_MAX);
    else if (is_finite(all)) r.sum = wave_sum(met.sum * rescale(met.mine, all, t));
    return r;
}

// A part of a row by a workgroup.
template <bool EXACT, int THREADS> __device__ __forceinline__ RowPart block_part(const Met<EXACT> &met, const Temper &t)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ float tops[WAVES];
    __shared__ RowPart sums[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float all = wave_top(met.top);
    if (lane == 0) tops[wave] = all;
    __syncthreads();
    all = tops[0];
#pragma unroll
    for (int w = 1; w < WAVES; w++) all = top_of(all, tops[w]);
    RowPart r = wave_part(met, all, t);
    if (lane == 0) sums[wave] = r;
    __syncthreads();
    r = sums[0];
#pragma unroll
    for (int w = 1; w < WAVES; w++) r.sum += sums[w].sum, r.first = sums[w].first < r.first ? sums[w].first : r.first;
    __syncthreads();
    return r;
}
template <bool EXACT, int THREADS, bool FP32> __device__ __forceinline__ RowPart part_of_row(const Row<FP32> row, int begin, int end, const Temper &t)
{
    return block_part<EXACT, THREADS>(meet_all<EXACT, THREADS>(row, begin, end, t, threadIdx.x), t);
}

// The sequence that row t belongs to: the number of those whose rows end at or before it, by 64 looks at a time.
__device__ __forceinline__ int sequence_of_row(const VerifyLaunch &a, int t, int lane)
{
    int b = 0, n = a.B;
    while (n > 0) {
        const int step = (n + 63) / 64, s = b + (lane + 1) * step - 1;
        const int ended = __popcll(__ballot(s < a.B && a.cu[s + 1] <= t));
        b += ended * step;
        n = step == 1 ? 0 : a.B - b < step ? a.B - b : step;
    }
    return b;
}

// The sequence that row t belongs to, its rows and what else of it a row needs; b is not below the number of sequences where there is none.
// Of up to 64 sequences, a wave's lanes, all is asked for at once: one trip to memory instead of three.  (With what the draws ask for early,
// see verify_draw_kernel: one sequence with four drafts 14.6 and 13.8 us, four without 10.2 and 9.7, 128 with four 95.7 and 92.3.)
struct Owner {
    int b, begin, end;
    float T;
    int64_t draft_row;           // of row t: its place in draft_logits, or -1
};
__device__ __forceinline__ Owner owner_of_row(const VerifyLaunch &a, int t, int lane)
{
    Owner o = {0, 0, 0, 1.f, -1};
    int first = 0;
    if (a.B <= 64) {
        const bool in = lane < a.B;
        const int next = in ? a.cu[lane + 1] : INT32_MAX, drafts = in && a.draft ? a.draft_rows[lane] : 0, none = a.cu[0];
        const float T = in && a.temperature ? a.temperature[lane] : 1.f;
        o.b = __popcll(__ballot(next <= t));
        if (o.b >= a.B) return o;
        o.begin = o.b ? __builtin_amdgcn_readlane(next, o.b - 1) : none, o.end = __builtin_amdgcn_readlane(next, o.b);
        o.T = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(T), o.b)), first = __builtin_amdgcn_readlane(drafts, o.b);
    } else {
        o.b = sequence_of_row(a, t, lane);
        if (o.b >= a.B) return o;
        o.begin = a.cu[o.b], o.end = a.cu[o.b + 1];
        if (a.temperature) o.T = a.temperature[o.b];
        if (a.draft) first = a.draft_rows[o.b];
    }
    const int64_t r = (int64_t)first + t - o.begin;
    o.draft_row = a.draft && r >= 0 && r < a.total_draft_rows ? r : -1;
    return o;
}

__device__ __forceinline__ const uint8_t *row_at(const void *logits, int64_t stride, int fp32, int64_t t)
{
    return (const uint8_t *)logits + t * stride * (fp32 ? 4 : 2);
}

// The draft row that belongs to row t of sequence b, or -1.
__device__ __forceinline__ int64_t draft_row_of(const VerifyLaunch &a, int b, int t)
{
    const int64_t r = (int64_t)a.draft_rows[b] + t - a.cu[b];
    return r >= 0 && r < a.total_draft_rows ? r : -1;
}

template <bool EXACT, int THREADS> __device__ __forceinline__ RowPart part_of(const uint8_t *at, int fp32, int begin, int end, const Temper &t)
{
    return fp32 ? part_of_row<EXACT, THREADS>(Row<true>{at}, begin, end, t) : part_of_row<EXACT, THREADS>(Row<false>{at}, begin, end, t);
}
template <bool EXACT> __device__ __forceinline__ RowPart part_by_wave(const uint8_t *at, int fp32, int begin, int end, const Temper &t)
{
    const int lane = threadIdx.x & 63;
    const Met<EXACT> met = fp32 ? meet_all<EXACT, 64>(Row<true>{at}, begin, end, t, lane) : meet_all<EXACT, 64>(Row<false>{at}, begin, end, t, lane);
    return wave_part(met, wave_top(met.top), t);
}
__device__ __forceinline__ int part_end(const VerifyLaunch &a, int k) { return k + 1 < a.parts ? (k + 1) * a.part_len : a.V; }

// A part of a target row, or of the draft's row that belongs to it, for each wave: the target's rows come first.
template <bool EXACT> __global__ __launch_bounds__(kVerifyThreads) void verify_rows_kernel(VerifyLaunch a)
{
    touch_lines(a);
    const int lane = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.opened) a.opened[0] = 0;
    const unsigned n = __builtin_amdgcn_readfirstlane(blockIdx.x * (kVerifyThreads / 64) + threadIdx.x / 64);
    const unsigned rows = n / (unsigned)a.parts, k = n % (unsigned)a.parts;
    const bool drafted = rows >= (unsigned)a.R;
    if (rows >= (unsigned)a.R * (a.draft ? 2u : 1u)) return;
    const int t = (int)(drafted ? rows - a.R : rows);
    const Owner of = owner_of_row(a, t, lane);
    if (of.b >= a.B || t < of.begin) return;
    const Temper temper = temper_from(of.T);
    const uint8_t *at = row_at(a.logits, a.stride, a.fp32, t);
    if (drafted) {
        if (t + 1 >= of.end || of.draft_row < 0 || temper.c == 0.0) return;
        at = row_at(a.draft, a.draft_stride, a.draft_fp32, of.draft_row);
    }
    const RowPart r = part_by_wave<EXACT>(at, drafted ? a.draft_fp32 : a.fp32, k * a.part_len, part_end(a, k), temper);
    if (lane == 0) (drafted ? a.draft_row : a.row)[(int64_t)t * a.parts + k] = r;
}

// The same for each workgroup, where there are few: a thread has two loads of a part at most, and a target's are asked for before it is
// known whose row it is.
__global__ __launch_bounds__(kVerifyThreads) void verify_few_rows_kernel(VerifyLaunch a)
{
    touch_lines(a);
    const int tid = threadIdx.x, lane = tid & 63;
    if (blockIdx.x == 0 && tid == 0 && a.opened) a.opened[0] = 0;
    const unsigned rows = blockIdx.x / (unsigned)a.parts, k = blockIdx.x % (unsigned)a.parts;
    const bool drafted = rows >= (unsigned)a.R;
    const int t = (int)(drafted ? rows - a.R : rows), end = part_end(a, k), i = k * a.part_len + tid * kVec, j = i + kVerifyThreads * kVec;
    float x[kVec], y[kVec];
    auto load = [&](const uint8_t *at, int fp32) {
        if (fp32) Row<true>{at}.load_some(x, i, end), Row<true>{at}.load_some(y, j, end);
        else Row<false>{at}.load_some(x, i, end), Row<false>{at}.load_some(y, j, end);
    };
    if (!drafted) load(row_at(a.logits, a.stride, a.fp32, t), a.fp32);
    const Owner of = owner_of_row(a, t, lane);
    if (of.b >= a.B || t < of.begin) return;
    const Temper temper = temper_from(of.T);
    if (drafted) {
        if (t + 1 >= of.end || of.draft_row < 0 || temper.c == 0.0) return;
        load(row_at(a.draft, a.draft_stride, a.draft_fp32, of.draft_row), a.draft_fp32);
    }
    Met<true> met;
    met.meet(x, i, temper, temper.c == 0.0), met.meet(y, j, temper, temper.c == 0.0);
    const RowPart r = block_part<true, kVerifyThreads>(met, temper);
    if (tid == 0) (drafted ? a.draft_row : a.row)[(int64_t)t * a.parts + k] = r;
}

// ---- decisions ----------------------------------------------------------------------------------------

// A row's parts together.  All lanes of a wave take part and have the result.
struct Whole {
    double sum;
    float top;                   // finite: the row has a distribution
    int first;
};
__device__ __forceinline__ Whole whole_row(const RowPart *part, RowPart r, int parts, const Temper &t, int lane) // r: part[lane]
{
    float top = r.top;
    for (int k = lane + 64; k < parts; k += 64) top = top_of(top, part[k].top);
    top = wave_top(top);
    Whole w = {0.0, top, INT32_MAX};
    if (!is_finite(top)) return w;
    for (int k = lane;;) {
        if (t.c == 0.0) w.first = r.top == top && r.first < w.first ? r.first : w.first;
        else if (is_finite(r.top)) w.sum += r.sum * rescale(r.top, top, t);
        k += 64;
        if (k >= parts) break;
        r = part[k];
    }
    if (t.c == 0.0) w.first = wave_least(w.first);
    else w.sum = wave_sum(w.sum);
    return w;
}

__device__ __forceinline__ float logit_at(const void *logits, int64_t stride, int fp32, int64_t t, int i)
{
    const uint8_t *const at = row_at(logits, stride, fp32, t);
    return fp32 ? Row<true>{at}[i] : Row<false>{at}[i];
}

// How a token is drawn from a row.
enum DrawFrom { kNothing, kTop, kRow, kRowWithout, kRest }; // no distribution; greedy; p; p without the draft; max(p - q, 0)
struct Draw {
    int from, x, row;            // x: the draft that was turned down, or the greedy token; row: of logits
    int q_row;                   // ... of draft_logits
    const uint8_t *p, *q;        // the rows
    float p_top, q_top;
    double p_scale, q_scale;     // p = weight(l, p_top) * p_scale
    Temper t;
};

// What row `row` says to its draft, and how a token is drawn from it if that does not stay: by the row's sums, what its draft is (x, no
// token: -1), the logits of that in the target's row and in the draft model's, and the draft model's row (-1: none, or greedy).  All lanes of a wave.
enum Verdict { kGoes, kStays, kUnsure };
struct Asked {
    int row, x;
    int64_t q_row;
    float l, m, u;
};
// What a row reads whose place is known, though not yet whose it is: its parts' sums, the draft model's, its draft and number.
struct Early {
    int row, x;
    float u;
    RowPart mine, yours;         // (yours: of whatever was there before, if the row has none; it is not used then)
};
__device__ __forceinline__ Early ask_early(const VerifyLaunch &a, int row, int lane)
{
    const RowPart none = {0.0, -INFINITY, INT32_MAX};
    Early e = {row, -1, 0.f, none, none};
    if (row + 1 < a.R) e.x = a.tokens[row + 1], e.u = a.u[row]; // (the batch's last row judges none)
    if (lane < a.parts) e.mine = a.row[(int64_t)row * a.parts + lane];
    if (a.draft && lane < a.parts) e.yours = a.draft_row[(int64_t)row * a.parts + lane];
    return e;
}
__device__ __forceinline__ Asked ask_row(const VerifyLaunch &a, int b, const Early &e, int end, const Temper &t)
{
    Asked r = {e.row, e.row + 1 < end ? e.x : -1, -1, 0.f, 0.f, e.u};
    if (r.x < 0 || r.x >= a.V) r.x = -1;
    if (r.x < 0) return r;
    r.l = logit_at(a.logits, a.stride, a.fp32, r.row, r.x);
    if (a.draft && t.c != 0.0) r.q_row = draft_row_of(a, b, r.row);
    if (r.q_row >= 0) r.m = logit_at(a.draft, a.draft_stride, a.draft_fp32, r.q_row, r.x);
    return r;
}
__device__ __forceinline__ Draw judge(const VerifyLaunch &a, const Asked &r, const Temper &t, const Whole &p, const Whole &q, double unsure, Verdict &says, double &lp)
{
    Draw d = {};
    d.row = r.row, d.x = r.x, d.t = t, d.p = row_at(a.logits, a.stride, a.fp32, r.row), d.p_top = p.top, d.p_scale = 1.0 / p.sum;
    says = kGoes, lp = 0.0;
    if (!is_finite(p.top)) {
        d.from = kNothing;
        return d;
    }
    if (t.c == 0.0) {
        d.from = kTop, says = r.x >= 0 && r.x == p.first ? kStays : kGoes, d.x = p.first;
        return d;
    }
    d.from = kRow;
    if (r.x < 0) return d;
    const double px = weight(r.l, p.top, t) / p.sum;
    lp = ((double)r.l - (double)p.top) * t.c / kLog2e - log(p.sum);
    double against = (double)r.u;
    if (!a.draft) d.from = kRowWithout;
    else {
        if (r.q_row < 0 || !is_finite(q.top)) return d;
        d.from = kRest, d.q_row = (int)r.q_row, d.q = row_at(a.draft, a.draft_stride, a.draft_fp32, r.q_row), d.q_top = q.top, d.q_scale = 1.0 / q.sum;
        against *= weight(r.m, q.top, t) / q.sum;
    }
    says = against < px ? kStays : kGoes;
    // (where px is 0 or the number is not positive, no error of the sums changes the answer)
    if (px > 0.0 && against > 0.0 && __builtin_fabs(against - px) <= unsure * px) says = kUnsure;
    return d;
}
// A part of a row and what is left of the border there.
struct Border {
    int part;                    // -1: no part has a share
    double at;
};
// The part that holds v times the sum of all parts' shares: the first that the running sum exceeds it in, or the last with any share
// where rounding (or a number of 1) leaves none.  share(k): part k's, asked for by lane k % 64, once if there are 64 parts at most.  A share
// below 2^-996 is none (its weights might all have vanished).  All lanes of a wave.
template <typename F> __device__ __forceinline__ Border border_of(F share, int parts, double v, int lane)
{
    auto some = [&](int k) {
        const double s = k < parts ? share(k) : 0.0;
        return s > 1e-300 ? s : 0.0;
    };
    double x = some(lane), total = wave_sum(x);
    for (int k = lane + 64; k < parts + lane; k += 64) total += wave_sum(some(k));
    const double border = v * total;
    Border found = {-1, 0.0};
    double run = 0.0;
    for (int base = 0;;) {
        const double scan = wave_scan(x), before = run + from_lane<0x138, 0xf>(scan); // (the lane before's; none for the first)
        const uint64_t any = __ballot(x > 0.0), past = __ballot(x > 0.0 && run + scan > border);
        if (any) {
            const int at = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
            found = {base + at, border - lane_of(before, at)};
        }
        if (past) break;
        run += last_lane(scan);
        base += 64;
        if (base >= parts) break;
        x = some(base + lane);
    }
    return found;
}

// The weight of a part of row p in parts of the whole row's.
__device__ __forceinline__ double share_of(const RowPart &r, const Draw &d)
{
    return is_finite(r.top) ? r.sum * rescale(r.top, d.p_top, d.t) * d.p_scale : 0.0;
}

// A row of sequence b by the sums that the first kernel left: the draw from it, what it says to its draft, and where v lies in it.
__device__ __forceinline__ Draw judge_row(const VerifyLaunch &a, int b, const Early &e, int end, const Temper &t, double v, int lane, double unsure, Verdict &says, double &lp, Border &border)
{
    const RowPart *const parts = a.row + (int64_t)e.row * a.parts, *const theirs = a.draft_row + (int64_t)e.row * a.parts;
    const Asked asked = ask_row(a, b, e, end, t);
    const Whole p = whole_row(parts, e.mine, a.parts, t, lane);
    Whole q = {1.0, -INFINITY, 0};
    if (asked.q_row >= 0) q = whole_row(theirs, e.yours, a.parts, t, lane);
    const Draw d = judge(a, asked, t, p, q, unsure, says, lp);
    if (d.from == kRow) border = border_of([&](int k) { return share_of(k == lane ? e.mine : parts[k], d); }, a.parts, v, lane);
    return d;
}

// A whole row, all over again in binary64, by a workgroup of the draws.
__device__ __forceinline__ Whole exact_row(const VerifyLaunch &a, const uint8_t *at, int fp32, const Temper &t)
{
    const RowPart r = part_of<true, kDrawThreads>(at, fp32, 0, a.V, t);
    return {r.sum, r.top, r.first};
}

// The rows of sequence b, as many at a time as there are waves, up to the first that keeps no draft: that one's draw.  The drafts that stay
// are written.  e: what was asked for before the rows were known.  The whole workgroup.
template <bool EXACT> __device__ __forceinline__ Draw decide(const VerifyLaunch &a, int b, int begin, int end, const Temper &t, double v, Early e, Border &border)
{
    __shared__ Draw draws[kDrawWaves];
    __shared__ Verdict verdict[kDrawWaves];
    __shared__ Border borders[kDrawWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int base = begin;; base += kDrawWaves) {
        const int row = base + wave;
        Verdict says = kGoes;
        double lp = 0.0;
        if (row < end) {
            Border in_row = {-1, 0.0};
            if (e.row != row) e = ask_early(a, row, lane);
            const Draw d = judge_row(a, b, e, end, t, v, lane, EXACT ? 0.0 : 4.0 * a.eps, says, lp, in_row);
            if (EXACT && says == kUnsure) says = kGoes;         // (equal: not less)
            if (lane == 0) draws[wave] = d, borders[wave] = in_row;
        }
        if (lane == 0) verdict[wave] = says;
        __syncthreads();
        int n = 0;
        for (;; n++) {
            while (n < kDrawWaves && verdict[n] == kStays) n++;
            if (EXACT || n == kDrawWaves || verdict[n] == kGoes) break;
            // too near to be told apart by sums of binary32 weights: a few in a hundred thousand
            const Draw d = draws[n];
            const Whole p = exact_row(a, d.p, a.fp32, t);
            const Whole q = d.from == kRest ? exact_row(a, d.q, a.draft_fp32, t) : Whole{1.0, -INFINITY, 0};
            Verdict sure;
            double unused;
            (void)judge(a, ask_row(a, b, ask_early(a, d.row, lane), end, t), t, p, q, 0.0, sure, unused);
            if (sure != kStays) break;
        }
        if (wave < n && lane == 0) {
            a.out[row] = a.tokens[row + 1];
            if (a.logprobs) a.logprobs[row] = (float)lp;
        }
        if (n < kDrawWaves) {                                   // (the last row keeps none, so there is one)
            border = borders[n];
            return draws[n];
        }
        __syncthreads();
    }
}

// ---- a token from its weights ---------------------------------------------------------------------------

// Weights of values i .. i + 7 (those at or past end are 0) in the sum that the token is drawn by, and the target's logits.
template <bool FP32, bool QFP32> __device__ __forceinline__ void weights(double (&w)[kVec], float (&x)[kVec], const Draw &d, int i, int end)
{
    float y[kVec];
    Row<FP32>{d.p}.load_some(x, i, end);
    if (d.from == kRest) {
        Row<QFP32>{d.q}.load_some(y, i, end);
#pragma unroll
        for (int j = 0; j < kVec; j++) {
#pragma clang fp contract(off)
            // (each product rounded by itself: where p and q are the same, nothing is left)
            const double r = weight(x[j], d.p_top, d.t) * d.p_scale - weight(y[j], d.q_top, d.t) * d.q_scale;
            w[j] = r > 0.0 ? r : 0.0;
        }
    } else {
#pragma unroll
        for (int j = 0; j < kVec; j++) w[j] = d.from == kRowWithout && i + j == d.x ? 0.0 : weight(x[j], d.p_top, d.t) * d.p_scale;
    }
}
__device__ __forceinline__ void weights_at(double (&w)[kVec], float (&x)[kVec], const VerifyLaunch &a, const Draw &d, int i, int end)
{
    if (a.fp32) a.draft_fp32 ? weights<true, true>(w, x, d, i, end) : weights<true, false>(w, x, d, i, end);
    else a.draft_fp32 ? weights<false, true>(w, x, d, i, end) : weights<false, false>(w, x, d, i, end);
}
// This thread's eight weights of part k, and their sum.
__device__ __forceinline__ double weights_of_part(double (&w)[kVec], float (&x)[kVec], const VerifyLaunch &a, const Draw &d, int k)
{
    weights_at(w, x, a, d, k * a.part_len + threadIdx.x * kVec, part_end(a, k));
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kVec; j++) sum += w[j];
    return sum;
}

struct DrawLds {
    double sums[kDrawWaves];
    int over[kDrawWaves], some[kDrawWaves];
};
__device__ __forceinline__ double block_sum(double x, DrawLds &lds)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds.sums[threadIdx.x >> 6] = x;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kDrawWaves; w++) total += lds.sums[w];
    return total;
}
// The thread whose share (mine) of a running sum over the workgroup holds the border: the first that the sum with it exceeds it in, or the
// last with any share where rounding (or a number of 1) leaves none; -1: no thread has any.  border: of the sum; v given: v times
// the sum of all.  before: the sum of the threads before this one.
__device__ __forceinline__ int holder(double mine, double &before, double &border, const double *v, DrawLds &lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const double scan = wave_scan(mine);
    __syncthreads();
    if (lane == 63) lds.sums[wave] = scan;
    __syncthreads();
    before = 0.0;
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kDrawWaves; w++) {
        if (w == wave) before = total;
        total += lds.sums[w];
    }
    if (v) border = *v * total;
    const uint64_t any = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && before + scan > border);
    const double up = from_lane<0x138, 0xf>(scan);              // (the lane before; none for the first)
    before += up;
    if (lane == 0) lds.over[wave] = past ? wave * 64 + __builtin_ctzll(past) : INT32_MAX, lds.some[wave] = any ? wave * 64 + 63 - __builtin_clzll(any) : -1;
    __syncthreads();
    int first = INT32_MAX, last = -1;
#pragma unroll
    for (int w = 0; w < kDrawWaves; w++) first = lds.over[w] < first ? lds.over[w] : first, last = lds.some[w] > last ? lds.some[w] : last;
    return first < INT32_MAX ? first : last;
}

// A token that was drawn, and its logit; -1: none, or the draw stays open.
struct Token {
    int id;
    float logit;
};
// The first value of the border's part at which the running sum of the part's weights passes the border; none where the sum is within `unsure` of
// the border at it or before it.
__device__ __forceinline__ Token token_of_part(const VerifyLaunch &a, const Draw &d, Border at, double unsure, DrawLds &lds)
{
    __shared__ Token token;
    const int tid = threadIdx.x, k = at.part;
    double border = at.at;
    if (k < 0) return {-1, 0.f};
    double w[kVec], before;
    float x[kVec];
    const double sum = weights_of_part(w, x, a, d, k);
    const int who = holder(sum, before, border, nullptr, lds);
    if (who < 0) return {-1, 0.f};
    if (tid == who) {
        double run = before, under = before;
        int which = -1;
        float logit = 0.f;
#pragma unroll
        for (int j = 0; j < kVec; j++)
            if (w[j] > 0.0 && (which < 0 || run <= border)) which = j, logit = x[j], under = run, run += w[j];
        const bool near = run - border <= unsure || border - under <= unsure;
        token = {which >= 0 && (unsure == 0.0 || !near) ? k * a.part_len + tid * kVec + which : -1, logit};
    }
    __syncthreads();
    return token;
}

// The token that v draws from p without the draft, by the parts' shares in p.  The part that the draft is in is added up anew: what is left
// of it may be far less than a difference of sums could say.  The whole workgroup.
template <typename F> __device__ __forceinline__ Token draw_without(const VerifyLaunch &a, const Draw &d, F share, double v, double unsure, DrawLds &lds)
{
    const int lane = threadIdx.x & 63, without = d.x / a.part_len;
    double w[kVec];
    float x[kVec];
    const double left = block_sum(weights_of_part(w, x, a, d, without), lds);
    const Border at = border_of([&](int k) { return k == without ? left : share(k); }, a.parts, v, lane);
    return token_of_part(a, d, at, unsure, lds);
}

__device__ __forceinline__ double number_of(const VerifyLaunch &a, int b)
{
    const double v = a.v[b];
    return v > 0.0 ? v < 1.0 ? v : 1.0 : 0.0;
}

// What comes out of sequence b, but for the drafts that stay.  The whole workgroup.
__device__ __forceinline__ void finish(const VerifyLaunch &a, int b, int begin, int end, const Draw &d, Token token)
{
    const int tid = threadIdx.x;
    if (tid == 0) {
        a.accepted[b] = d.row - begin;
        if (a.next) a.next[b] = token.id;
        a.out[d.row] = token.id;
        if (a.logprobs) {
            double lp = d.from == kTop ? 0.0 : __builtin_nan("");
            if (d.from != kTop && token.id >= 0) lp = ((double)token.logit - (double)d.p_top) * d.t.c / kLog2e + log(d.p_scale);
            a.logprobs[d.row] = (float)lp;
        }
    }
    for (int i = d.row + 1 + tid; i < end; i += kDrawThreads) {
        a.out[i] = -1;
        if (a.logprobs) a.logprobs[i] = 0.f;
    }
}

// Which drafts stay, and the token behind them where the row's sums tell it: a workgroup for each sequence.  What is left open: draws
// from p - q, and those that binary32 sums do not settle.
template <bool EXACT> __global__ __launch_bounds__(kDrawThreads) void verify_draw_kernel(VerifyLaunch a)
{
    touch_lines(a);
    __shared__ DrawLds lds;
    const int tid = threadIdx.x, b = blockIdx.x;
    // (where sequences have as many rows each, this wave's row is known before the offsets are)
    const int64_t likely = (int64_t)b * (a.R / a.B) + (tid >> 6);
    Early e = {};
    e.row = -1;
    if (likely < a.R) e = ask_early(a, (int)likely, tid & 63);
    const int begin = a.cu[b], end = a.cu[b + 1];
    if (begin < 0 || end > a.R || begin >= end) {
        if (tid == 0) {
            a.accepted[b] = 0;
            if (a.next) a.next[b] = -1;
        }
        return;
    }
    const float T = a.temperature ? a.temperature[b] : 1.f;
    const double v = number_of(a, b), unsure = EXACT ? 0.0 : 3.0 * a.eps; // (prefixes and totals are off by eps of the row each)
    const Temper t = temper_from(T);
    Border at;
    const Draw d = decide<EXACT>(a, b, begin, end, t, v, e, at);
    Token token = {d.from == kTop ? d.x : -1, 0.f};
    if (d.from == kRow) token = token_of_part(a, d, at, unsure, lds);
    else if (d.from == kRowWithout) {
        const RowPart *const parts = a.row + (int64_t)d.row * a.parts;
        token = draw_without(a, d, [&](int k) { return share_of(parts[k], d); }, v, unsure, lds);
        if (EXACT && token.id < 0) {                            // nothing is left: p
            Draw p = d;
            p.from = kRow;
            token = token_of_part(a, p, border_of([&](int k) { return share_of(parts[k], d); }, a.parts, v, tid & 63), 0.0, lds);
        }
    }
    if (d.from == kRest || (!EXACT && token.id < 0 && d.from != kNothing)) {
        // (in any order: draws do not look at each other)
        if (tid == 0) a.open[atomicAdd(a.opened, 1)] = {b, d.from, d.row, d.x, d.q_row, 0, T, d.p_top, d.q_top, d.p_scale, d.q_scale};
    } else finish(a, b, begin, end, d, token);
}

// A sum for whichever workgroup draws, and whether that is this one: the last of an open draw's workgroups, one a part.  The sum goes past
// the caches to where every die sees it, is waited for, and only then counts; it is read the same way.  (A release and an acquire
// would write back and drop the die's whole cache for these eight bytes: 55 us instead of 27 for 1 700 workgroups, 115 instead of 43 for 3 000.)
__device__ __forceinline__ bool last_to_publish(const VerifyLaunch &a, OpenDraw &o, double *at, double sum)
{
    __shared__ int arrived;
    if (threadIdx.x == 0) {
        __hip_atomic_store(at, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        arrived = __hip_atomic_fetch_add(&o.arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return arrived == a.parts - 1;
}
__device__ __forceinline__ double published(const double *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Every part of every open draw, an item to a workgroup at a time.
template <typename F> __device__ __forceinline__ void every_item(const VerifyLaunch &a, F f)
{
    unsigned at = blockIdx.x / (unsigned)a.parts, k = blockIdx.x % (unsigned)a.parts;
    OpenDraw o = a.open[at];                                    // (there is one, if of nothing: asked for beside their number)
    const unsigned n = (unsigned)a.opened[0] * (unsigned)a.parts;
    for (unsigned j = blockIdx.x; j < n;) {
        f(o, (int)at, (int)k);
        j += gridDim.x, at = j / (unsigned)a.parts, k = j % (unsigned)a.parts;
        if (j < n) o = a.open[at];
        __syncthreads();
    }
}

// An open draw by what the draws' kernel knew of its rows.
__device__ __forceinline__ Draw open_draw(const VerifyLaunch &a, const OpenDraw &o)
{
    Draw d = {};
    d.from = o.from, d.row = o.row, d.x = o.x, d.q_row = o.q_row, d.t = temper_from(o.T), d.p = row_at(a.logits, a.stride, a.fp32, o.row);
    d.p_top = o.p_top, d.p_scale = o.p_scale, d.q_top = o.q_top, d.q_scale = o.q_scale;
    if (o.from == kRest) d.q = row_at(a.draft, a.draft_stride, a.draft_fp32, o.q_row);
    return d;
}
// Its token, by the shares of its row's parts (and of p's parts, where nothing is left of p - q, or without the draft).  The whole workgroup.
template <typename F, typename G> __device__ __forceinline__ Token close_draw(const VerifyLaunch &a, Draw &d, F share, G share_in_p, double v, DrawLds &lds)
{
    Token token = {-1, 0.f};
    if (d.from == kRowWithout) token = draw_without(a, d, share, v, 0.0, lds);
    else if (d.from == kRest) token = token_of_part(a, d, border_of(share, a.parts, v, threadIdx.x & 63), 0.0, lds);
    if (token.id >= 0) return token;
    d.from = kRow;
    return token_of_part(a, d, border_of(share_in_p, a.parts, v, threadIdx.x & 63), 0.0, lds);
}

// Few open draws, from p: its sums anew, in binary64; the last workgroup to add up its part draws.
__global__ __launch_bounds__(kDrawThreads) void verify_again_kernel(VerifyLaunch a)
{
    touch_lines(a);
    __shared__ DrawLds lds;
    every_item(a, [&](const OpenDraw &o, int at, int k) {
        Draw d = open_draw(a, o);
        const double v = number_of(a, o.b);                     // (asked for before the sums are there)
        const RowPart p = part_of<true, kDrawThreads>(d.p, a.fp32, k * a.part_len, part_end(a, k), d.t);
        double *const sums = a.rest + (int64_t)o.row * a.parts;
        if (!last_to_publish(a, a.open[at], sums + k, share_of(p, d))) return;
        const int lane = threadIdx.x & 63;
        const double mine = lane < a.parts ? published(sums + lane) : 0.0;
        double all = mine;
        for (int j = lane + 64; j < a.parts; j += 64) all += published(sums + j);
        auto share = [&](int j) { return j == lane ? mine : published(sums + j); };
        // the log-probability is of these sums, too, which come to 1 + more: 1 / (1 + more) to its third order, 10^-16
        const double more = wave_sum(all) - 1.0, scale = d.p_scale * __builtin_fma(more, more - 1.0, 1.0);
        const Token token = close_draw(a, d, share, share, v, lds);
        d.p_scale = scale;
        finish(a, o.b, a.cu[o.b], a.cu[o.b + 1], d, token);
    });
}
// ... from p - q, whose sums are binary64: what is left of it, in the same way.
__global__ __launch_bounds__(kDrawThreads) void verify_rest_kernel(VerifyLaunch a)
{
    touch_lines(a);
    __shared__ DrawLds lds;
    every_item(a, [&](const OpenDraw &o, int at, int k) {
        Draw d = open_draw(a, o);
        double w[kVec];
        float x[kVec];
        const double sum = block_sum(weights_of_part(w, x, a, d, k), lds);
        double *const sums = a.rest + (int64_t)o.row * a.parts;
        if (!last_to_publish(a, a.open[at], sums + k, sum)) return;
        const RowPart *const parts = a.row + (int64_t)o.row * a.parts;
        const Token token = close_draw(a, d, [&](int k) { return published(sums + k); }, [&](int k) { return share_of(parts[k], d); }, number_of(a, o.b), lds);
        finish(a, o.b, a.cu[o.b], a.cu[o.b + 1], d, token);
    });
}

// Many open draws, whose sums are binary32: all of it anew, in binary64, and in one pass over p and q, though their scales are only known
// when it is over.  With a and b the weights of a value by the scales at hand, p = alpha a and q = beta b, alpha and beta within eps of 1:
//   sum max(p - q, 0) = alpha sum max(a - b, 0) + (alpha - beta) sum_{a > b} b,
// but for values where p and q are so near each other that the scales decide which is larger, |a - b| < 4 eps b: each is off by 6 eps b
// at most.  The sum of those b says how much all may be off, which is next to nothing, or where models agree over much of a row, a doubt
// that verify_close_kernel settles.  A workgroup has a part.  (128, 256, 512 threads: 97.5, 96.0, 99.2 us of 128 x 5 rows of 152 064 bf16 values with a
// draft model's.)
constexpr int kOpenThreads = 256;
template <bool FP32, bool QFP32> __device__ __forceinline__ void add_up(OpenPart &s, const Draw &d, double near, int i, int end)
{
    float x[kVec], y[kVec];
    Row<FP32>{d.p}.load_some(x, i, end), Row<QFP32>{d.q}.load_some(y, i, end);
    bool any = false;
    double a[kVec], b[kVec];
#pragma unroll
    for (int j = 0; j < kVec; j++) {
#pragma clang fp contract(off)
        const double p = weight(x[j], d.p_top, d.t), q = weight(y[j], d.q_top, d.t);
        s.p += p, s.q += q;
        a[j] = p * d.p_scale, b[j] = q * d.q_scale;
        const double more = a[j] - b[j];
        s.more += __builtin_fmax(more, 0.0);
        s.under += more > 0.0 ? b[j] : 0.0;
        any |= __builtin_fabs(more) < near * b[j];
    }
    if (!__any(any)) return;
#pragma unroll
    for (int j = 0; j < kVec; j++) s.near += __builtin_fabs(a[j] - b[j]) < near * b[j] ? b[j] : 0.0;
}
__global__ __launch_bounds__(kOpenThreads) void verify_left_kernel(VerifyLaunch a)
{
    touch_lines(a);
    __shared__ OpenPart waves[kOpenThreads / 64];
    const int tid = threadIdx.x;
    every_item(a, [&](const OpenDraw &o, int at, int k) {
        const Draw d = open_draw(a, o);
        const int end = part_end(a, k);
        const double near = 4.0 * a.eps;
        OpenPart s = {};
        for (int i = k * a.part_len + tid * kVec; i < end; i += kOpenThreads * kVec) {
            if (d.from != kRest) {
                float x[kVec];
                if (a.fp32) Row<true>{d.p}.load_some(x, i, end);
                else Row<false>{d.p}.load_some(x, i, end);
#pragma unroll
                for (int j = 0; j < kVec; j++) s.p += weight(x[j], d.p_top, d.t);
            } else if (a.fp32) a.draft_fp32 ? add_up<true, true>(s, d, near, i, end) : add_up<true, false>(s, d, near, i, end);
            else a.draft_fp32 ? add_up<false, true>(s, d, near, i, end) : add_up<false, false>(s, d, near, i, end);
        }
        s = {wave_sum(s.p), wave_sum(s.q), wave_sum(s.more), wave_sum(s.under), wave_sum(s.near)};
        if ((tid & 63) == 0) waves[tid >> 6] = s;
        __syncthreads();
        if (tid) return;
#pragma unroll
        for (int w = 1; w < kOpenThreads / 64; w++) s.p += waves[w].p, s.q += waves[w].q, s.more += waves[w].more, s.under += waves[w].under, s.near += waves[w].near;
        a.left[(int64_t)at * a.parts + k] = s;
    });
}
// The tokens, a draw to a workgroup.
__global__ __launch_bounds__(kDrawThreads) void verify_close_kernel(VerifyLaunch a)
{
    touch_lines(a);
    __shared__ DrawLds lds;
    const int lane = threadIdx.x & 63;
    const OpenDraw o = a.open[blockIdx.x];
    const OpenPart *const parts = a.left + (int64_t)blockIdx.x * a.parts;
    const OpenPart mine = lane < a.parts ? parts[lane] : OpenPart{}; // (before it is known that there is such a draw)
    if ((int)blockIdx.x >= a.opened[0]) return;
    Draw d = open_draw(a, o);
    OpenPart all = mine;
    for (int k = lane + 64; k < a.parts; k += 64) all.p += parts[k].p, all.q += parts[k].q, all.near += parts[k].near;
    const double p_scale = 1.0 / wave_sum(all.p), q_scale = 1.0 / wave_sum(all.q), v = number_of(a, o.b);
    const double alpha = p_scale / d.p_scale, skew = alpha - q_scale / d.q_scale, unsure = 13.0 * a.eps * wave_sum(all.near);
    d.p_scale = p_scale, d.q_scale = q_scale;
    auto part = [&](int k) { return k == lane ? mine : parts[k]; };
    auto share_in_p = [&](int k) { return part(k).p * p_scale; };
    Token token = {-1, 0.f};
    if (d.from == kRest) {
        const Border at = border_of([&](int k) { const OpenPart s = part(k); return alpha * s.more + skew * s.under; }, a.parts, v, lane);
        token = token_of_part(a, d, at, unsure, lds);
        if (token.id < 0) {                                     // in doubt, or nothing is left: part by part
            double *const sums = a.rest + (int64_t)o.row * a.parts;
            for (int k = 0; k < a.parts; k++) {
                double w[kVec];
                float x[kVec];
                const double sum = block_sum(weights_of_part(w, x, a, d, k), lds);
                if (threadIdx.x == 0) sums[k] = sum;
            }
            __syncthreads();
            token = close_draw(a, d, [&](int k) { return sums[k]; }, share_in_p, v, lds);
        }
    } else token = close_draw(a, d, share_in_p, share_in_p, v, lds);
    finish(a, o.b, a.cu[o.b], a.cu[o.b + 1], d, token);
}

// Rows are cut into parts of 4096 values: a draw then looks at eight for each thread.
constexpr int kPart = kDrawThreads * kVec;
static int parts_of(int V) { return (V + kPart - 1) / kPart; }

// A row's parts go to a wave each where those are six for every compute unit, to a workgroup each where there are fewer.  (us of a
// call, waves and workgroups: 1 216 parts 14.1, 13.1; 1 824 parts 14.5, 15.4; 3 840 24.3, 26.7.)
// Whether all sums are binary64 from the start: binary32 sums are up to twice as fast, but leave draws open, which take another kernel or
// two; and their draws' kernel needs 154 registers, so that a compute unit holds one workgroup of it, not two, which tells where there is
// one for few logits (8 750 rows of 8 000: 185 us against 100).  With a draft model draws from p - q are open either way, and cost less after
// binary32 sums.  Binary32 logits are twice the bytes: there is less to gain.
// So: few logits for bf16, five times as many for binary32, and as many again for every kSeqsOfFew sequences; with a draft model's logits,
// both counted, half as many and five quarters.  Measured, us of a call with binary64 and with binary32 sums first, and the draws then open:
//   one row a sequence, bf16    92 x 152064   21.1   22.0  0-3     145 x 152064   26.5   26.7  1-5     329 x 152064   50.4   42.5   3-6
//                              280 x 100000   31.1   32.9  3-7     360 x 100000   38.2   37.4  4-10    557 x 50257    38.0   41.2   6-7
//                              995 x 50257    57.8   55.7  10-12  1125 x 32000    47.0   52.9  3-6    3125 x 32000   118.6  114.6  13-28
//                             8750 x 8000    162.1  221.5  11-14
//   ... binary32               395 x 152064   61.3   66.9  7-12    592 x 152064   90.6   92.4  10-16   723 x 152064  108.8  106.3  13-16
//   five rows, bf16             18 x 152064   23.9   21.6  0-1      24 x 152064   27.3   27.7  0-2      37 x 152064   33.2   31.1   0-3
//   ... binary32               298 x 50257    82.5   86.3  3-5     438 x 50257   112.3  110.2  4-7
//   five rows, draft, bf16       4 x 152064   24.8   25.3  1-2       6 x 152064   24.5   22.2  0-3      29 x 152064   53.8   41.6   7-9
//                               55 x 152064   83.7   54.6  12-15    28 x 32000    28.7   27.0  4-12
//   ... binary32                12 x 152064   33.2   35.6  0-6      15 x 152064   41.2   40.8  3-6      55 x 152064   90.0   78.9  11-16
constexpr double kSeqsOfFew = 680.0;
static void verify_shape(VerifyLaunch &a, int num_cus, int64_t few, bool drafted)
{
    const int64_t rows = (int64_t)a.R * (drafted ? 2 : 1);
    a.num_cus = num_cus;
    a.part_len = kPart;
    a.parts = parts_of(a.V);
    a.alone = rows * a.parts >= (int64_t)num_cus * 6;
    const double times = drafted ? a.fp32 ? 1.25 : 0.5 : (a.fp32 ? 5.0 : 1.0) + a.B / kSeqsOfFew;
    a.exact = (double)(rows * a.V) <= (double)few * times;
    // The error of a sum of weights as weight32 gives them, in parts of the row's whole sum W: a weight w is off by (3 ln 2 |y| + 2) 2^-24
    // of it and a sum of eight by 3 2^-24; y is against the thread's value, which is at most 8 / c below one it met: |y| is at most 8
    // more than against the row's largest.  Against that, log2(W) + sum(w |y|) / W is the entropy of the row in bits, at most log2(V),
    // and W >= 1: so sum(w |y|) <= log2(V) W.  All together (3 ln 2 (log2(V) + 8) + 5) 2^-24, and a twentieth more for second orders.
    int bits = 0;
    while ((int64_t)1 << bits < a.V) bits++;
    a.eps = 1.05 * (2.08 * (bits + 8) + 5.0) * 0x1p-24;
}

size_t carve_verify(VerifyLaunch &a, int num_cus, int64_t few, bool drafted, void *base)
{
    verify_shape(a, num_cus, few, drafted);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *const p = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    const size_t parts = (size_t)a.R * a.parts;
    a.row = (RowPart *)take(parts * sizeof(RowPart));
    if (drafted) a.draft_row = (RowPart *)take(parts * sizeof(RowPart));
    if (drafted || !a.exact) {
        a.rest = (double *)take(parts * sizeof(double));
        a.opened = (int32_t *)take(sizeof(int32_t));
        a.open = (OpenDraw *)take((size_t)a.B * sizeof(OpenDraw));
        if (drafted && !a.exact) a.left = (OpenPart *)take((size_t)a.B * a.parts * sizeof(OpenPart));
    }
    return at;
}

// (a launch has less than 2^32 threads)
bool verify_fits(int32_t B, int32_t R, int32_t V, bool drafted)
{
    const int64_t parts = parts_of(V);
    return R * parts * (drafted ? 2 : 1) * 64 < (int64_t)1 << 32 && B * parts < (int64_t)1 << 32;
}

hipError_t launch_verify(const VerifyLaunch &a, hipStream_t s)
{
    const unsigned rows = (unsigned)a.R * (unsigned)a.parts * (a.draft ? 2u : 1u), each = kVerifyThreads / 64;
    const int64_t items = (int64_t)a.B * a.parts, most = 2 * a.num_cus, lots = 16 * a.num_cus;
    const dim3 seqs((unsigned)a.B), threads(kDrawThreads), open((unsigned)(items < most ? items : most)), many((unsigned)(items < lots ? items : lots));
    if (a.R > 0) {
        const dim3 grid((rows + each - 1) / each);
        if (!a.exact) hipLaunchKernelGGL(verify_rows_kernel<false>, grid, dim3(kVerifyThreads), 0, s, a);
        else if (a.alone) hipLaunchKernelGGL(verify_rows_kernel<true>, grid, dim3(kVerifyThreads), 0, s, a);
        else hipLaunchKernelGGL(verify_few_rows_kernel, dim3(rows), dim3(kVerifyThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.exact) hipLaunchKernelGGL(verify_draw_kernel<true>, seqs, threads, 0, s, a);
    else hipLaunchKernelGGL(verify_draw_kernel<false>, seqs, threads, 0, s, a);
    if (!a.opened || a.R == 0) return hipGetLastError();        // (nothing is left open)
    if (!a.draft) hipLaunchKernelGGL(verify_again_kernel, open, threads, 0, s, a);
    else if (a.exact) hipLaunchKernelGGL(verify_rest_kernel, open, threads, 0, s, a);
    else {
        hipLaunchKernelGGL(verify_left_kernel, many, dim3(kOpenThreads), 0, s, a);
        hipLaunchKernelGGL(verify_close_kernel, seqs, threads, 0, s, a);
    }
    return hipGetLastError();
}

} // namespace ra
