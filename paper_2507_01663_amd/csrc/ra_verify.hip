// gfx950 kernels of the verification of drafted tokens and the choice of next ones.
//
// p = softmax(l / T) over rows of many thousand logits, from which one token is drawn by a running sum.  The borders of that sum
// decide, and there are as many as tokens: with binary32 weights each moves by some 2^-26 of the whole, which over 150 000 of them
// changes one token in a few hundred; so weights, sums and comparisons are binary64, at the same rate as binary32 on this machine.
#include "ra_device.h"
#include "ra_step.h"

namespace ra {

constexpr int kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / 64;
constexpr int kVec = 8;                                          // values that a lane loads at a time
constexpr double kLog2e = 1.4426950408889634074;

// What a row's weights are made with: 2^((l - top) * c).
struct Temper {
    double c;                    // log2(e) / T; 0: greedy
    double low;                  // differences at or below this weigh nothing: 2^-1100
    float cf;
};
__device__ __forceinline__ Temper temper_of(const VerifyLaunch &a, int b)
{
    float T = a.temperature ? a.temperature[b] : 1.f;
    Temper t;
    if (!(T > 0.f)) return {0.0, 0.0, 0.f};
    T = T < 1e-30f ? 1e-30f : T > 1e30f ? 1e30f : T;
    t.c = kLog2e / (double)T, t.low = -1100.0 / t.c, t.cf = (float)t.c;
    return t;
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
    const double d = (double)l - top;
    return power(d > t.low ? d : t.low, t.c);
}

// The larger of the two, or NaN if one is.
__device__ __forceinline__ float top_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <bool FP32> struct Row {
    const uint8_t *at;
    static constexpr int kBytes = FP32 ? 4 : 2;
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (FP32) return ((const float *)at)[i];
        else return __uint_as_float((uint32_t)((const uint16_t *)at)[i] << 16);
    }
    // Values i .. i + 7.  (A row begins at any element: the load is of no alignment but that.)
    __device__ __forceinline__ void load(float (&x)[kVec], int i) const
    {
        if constexpr (FP32) {
            __builtin_memcpy(x, at + (size_t)i * 4, 32);
        } else {
            uint32_t w[4];
            __builtin_memcpy(w, at + (size_t)i * 2, 16);
#pragma unroll
            for (int j = 0; j < 4; j++) x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
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

// The largest of values [begin, end) of a row and the sum of their weights against it; of a greedy row, the first of the largest.  A thread's
// sum stands against the first value that it met (binary64 has room for weights of 2^500); the block's against the largest.
template <bool FP32> __device__ RowPart part_of_row(const Row<FP32> row, int begin, int end, const Temper &t)
{
    __shared__ float tops[kVerifyWaves];
    __shared__ double part_sums[kVerifyWaves];
    __shared__ int firsts[kVerifyWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool greedy = t.c == 0.0;
    float top = -INFINITY, mine = -__FLT_MAX__;
    int first = INT32_MAX;
    double sum = 0.0, against = mine;
    for (int i = begin + tid * kVec; i < end; i += kVerifyThreads * kVec) {
        float x[kVec];
        row.load_some(x, i, end);
        float m = x[0];
#pragma unroll
        for (int j = 1; j < kVec; j++) m = top_of(m, x[j]);
        if (greedy) {
            if (m > top)
#pragma unroll
                for (int j = kVec - 1; j >= 0; j--)
                    if (x[j] == m) first = i + j;
        } else {
            if ((m - mine) * t.cf > 500.f) {                    // (also the first time)
                sum *= exp2(((double)mine - (double)m) * t.c);
                mine = m, against = m;
            }
#pragma unroll
            for (int j = 0; j < kVec; j++) sum += weight(x[j], against, t);
        }
        top = top_of(top, m);
    }
    float all = top;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) all = top_of(all, __shfl_xor(all, d));
    if (lane == 0) tops[wave] = all;
    __syncthreads();
    all = tops[0];
#pragma unroll
    for (int w = 1; w < kVerifyWaves; w++) all = top_of(all, tops[w]);
    sum = is_finite(all) ? sum * exp2(((double)mine - (double)all) * t.c) : 0.0;
    if (top != all) first = INT32_MAX;
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        sum += __shfl_xor(sum, d);
        const int other = __shfl_xor(first, d);
        first = other < first ? other : first;
    }
    if (lane == 0) part_sums[wave] = sum, firsts[wave] = first;
    __syncthreads();
    RowPart r = {part_sums[0], all, firsts[0]};
#pragma unroll
    for (int w = 1; w < kVerifyWaves; w++) r.sum += part_sums[w], r.first = firsts[w] < r.first ? firsts[w] : r.first;
    return r;
}

// The sequence that row t belongs to: the number of those whose rows end at or before it.
__device__ __forceinline__ int sequence_of_row(const VerifyLaunch &a, int t, int lane)
{
    int b = 0;
    for (int base = 0; base < a.B; base += 64) {
        const int s = base + lane;
        const int n = __popcll(__ballot(s < a.B && a.cu[s + 1] <= t));
        b += n;
        if (n < 64) break;
    }
    return b;
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

// A part of a target row, or of the draft's row that belongs to it: the workgroups of the target's rows come first.
__global__ __launch_bounds__(kVerifyThreads) void verify_rows_kernel(VerifyLaunch a)
{
    const unsigned rows = blockIdx.x / (unsigned)a.parts, k = blockIdx.x % (unsigned)a.parts;
    const bool drafted = rows >= (unsigned)a.R;
    const int t = (int)(drafted ? rows - a.R : rows), lane = threadIdx.x & 63;
    const int b = sequence_of_row(a, t, lane);
    if (b >= a.B || t < a.cu[b]) return;
    const Temper temper = temper_of(a, b);
    const int begin = (int)k * a.part_len, end = begin + a.part_len < a.V ? begin + a.part_len : a.V;
    RowPart r;
    if (!drafted) {
        const uint8_t *const at = row_at(a.logits, a.stride, a.fp32, t);
        r = a.fp32 ? part_of_row(Row<true>{at}, begin, end, temper) : part_of_row(Row<false>{at}, begin, end, temper);
    } else {
        const int64_t d = draft_row_of(a, b, t);
        if (t + 1 >= a.cu[b + 1] || d < 0 || temper.c == 0.0) return;
        const uint8_t *const at = row_at(a.draft, a.draft_stride, a.draft_fp32, d);
        r = a.draft_fp32 ? part_of_row(Row<true>{at}, begin, end, temper) : part_of_row(Row<false>{at}, begin, end, temper);
    }
    if (threadIdx.x == 0) (drafted ? a.draft_row : a.row)[(int64_t)t * a.parts + k] = r;
}

// ---- decisions ----------------------------------------------------------------------------------------

// A row's parts together.  All lanes of a wave take part and have the result.
struct Whole {
    double sum;
    float top;                   // finite: the row has a distribution
    int first;
};
__device__ __forceinline__ Whole whole_row(const RowPart *part, int parts, const Temper &t, int lane)
{
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 64) top = top_of(top, part[k].top);
#pragma unroll
    for (int d = 32; d > 0; d /= 2) top = top_of(top, __shfl_xor(top, d));
    double sum = 0.0;
    int first = INT32_MAX;
    if (is_finite(top))
        for (int k = lane; k < parts; k += 64) {
            const RowPart r = part[k];
            if (r.top == top && r.first < first) first = r.first;
            if (is_finite(r.top)) sum += r.sum * exp2(((double)r.top - (double)top) * t.c);
        }
#pragma unroll
    for (int d = 32; d > 0; d /= 2) {
        sum += __shfl_xor(sum, d);
        const int other = __shfl_xor(first, d);
        first = other < first ? other : first;
    }
    return {sum, top, first};
}

__device__ __forceinline__ float logit_at(const void *logits, int64_t stride, int fp32, int64_t t, int i)
{
    const uint8_t *const at = row_at(logits, stride, fp32, t);
    return fp32 ? Row<true>{at}[i] : Row<false>{at}[i];
}

// How a token is drawn from a row.
enum DrawFrom { kNothing, kTop, kRow, kRowWithout, kRest }; // no distribution; greedy; p; p without the draft; max(p - q, 0)
struct Draw {
    int from, x, dfp32;          // x: the draft that was turned down
    const uint8_t *p, *q;        // the rows
    double p_top, p_scale, q_top, q_scale; // p = weight(l, p_top) * p_scale
    Temper t;
};

// The weight of value i in the sum that the token is drawn by.
template <bool FP32, bool QFP32> struct Weights {
    Draw d;
    __device__ __forceinline__ double operator()(int i) const
    {
#pragma clang fp contract(off)
        // (each product rounded by itself: where p and q are the same, nothing is left)
        double w = weight(Row<FP32>{d.p}[i], d.p_top, d.t) * d.p_scale;
        if (d.from == kRest) {
            w -= weight(Row<QFP32>{d.q}[i], d.q_top, d.t) * d.q_scale;
            w = w > 0.0 ? w : 0.0;
        }
        return d.from == kRowWithout && i == d.x ? 0.0 : w;
    }
};

__device__ __forceinline__ double block_sum_before(double x, double *lds, double &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    double before = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kVerifyWaves; w++) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    __syncthreads();
    return before + s - x;
}

// The token: the first value at which the running sum passes v times the whole.  Every thread has one stretch of the row; the one
// that holds the border walks it again.
template <typename W> __device__ int draw(const W &w, int V, double v, bool &nothing)
{
    __shared__ double lds[kVerifyWaves];
    __shared__ int found, last;
    const int tid = threadIdx.x, len = (V + kVerifyThreads - 1) / kVerifyThreads;
    const int begin = tid * len < V ? tid * len : V, end = begin + len < V ? begin + len : V;
    if (tid == 0) found = INT32_MAX, last = -1;
    double mine = 0.0, total;
    for (int i = begin; i < end; i++) mine += w(i);
    const double before = block_sum_before(mine, lds, total);
    const double border = v * total;
    if (mine > 0.0) atomicMax(&last, tid);
    if (before <= border && before + mine > border) atomicMin(&found, tid);
    __syncthreads();
    nothing = !(total > 0.0);
    const int who = found < last ? found : last;
    __syncthreads();
    if (tid == who) {
        double run = before;
        int token = -1;
        for (int i = begin; i < end; i++) {
            const double x = w(i);
            if (!(x > 0.0)) continue;
            token = i, run += x;
            if (run > border) break;
        }
        found = token;
    }
    __syncthreads();
    return found;
}

template <bool FP32, bool QFP32> __device__ int draw_from(Draw &d, int V, double v)
{
    bool nothing = false;
    int token = draw(Weights<FP32, QFP32>{d}, V, v, nothing);
    if (nothing) {
        __syncthreads();
        d.from = kRow;
        token = draw(Weights<FP32, QFP32>{d}, V, v, nothing);
    }
    return token;
}

// One workgroup for each sequence: which drafts stay, and the token behind them.
__global__ __launch_bounds__(kVerifyThreads) void verify_draw_kernel(VerifyLaunch a)
{
    __shared__ Draw shared;
    __shared__ int kept, done;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int begin = a.cu[b], end = a.cu[b + 1];
    if (begin < 0 || end > a.R || begin >= end) {
        if (tid == 0) {
            a.accepted[b] = 0;
            if (a.next) a.next[b] = -1;
        }
        return;
    }
    const Temper t = temper_of(a, b);
    if (tid == 0) done = 0;
    __syncthreads();
    // rows one after the other, until one accepts no draft
    for (int row = begin; row < end; row++) {
        if (wave == 0) {
            const Whole p = whole_row(a.row + (int64_t)row * a.parts, a.parts, t, lane);
            const bool last = row + 1 == end;
            const int x = last ? -1 : a.tokens[row + 1];
            const bool token = x >= 0 && x < a.V;
            Draw d = {};
            d.x = x, d.t = t, d.p = row_at(a.logits, a.stride, a.fp32, row), d.p_top = p.top, d.p_scale = 1.0 / p.sum;
            bool stays = false;
            double lp = 0.0;
            if (!is_finite(p.top)) d.from = kNothing;
            else if (t.c == 0.0) {
                d.from = kTop, stays = token && x == p.first;
                d.x = p.first;
            } else {
                d.from = kRow;
                double px = 0.0;
                if (token) {
                    const float l = logit_at(a.logits, a.stride, a.fp32, row, x);
                    px = weight(l, p.top, t) / p.sum;
                    lp = ((double)l - (double)p.top) * t.c / kLog2e - log(p.sum);
                }
                if (token && !a.draft) {
                    stays = (double)a.u[row] < px;
                    d.from = kRowWithout;
                } else if (token) {
                    const int64_t r = draft_row_of(a, b, row);
                    if (r >= 0) {
                        const Whole q = whole_row(a.draft_row + (int64_t)row * a.parts, a.parts, t, lane);
                        if (is_finite(q.top)) {
                            d.from = kRest, d.dfp32 = a.draft_fp32, d.q = row_at(a.draft, a.draft_stride, a.draft_fp32, r);
                            d.q_top = q.top, d.q_scale = 1.0 / q.sum;
                            const double qx = weight(logit_at(a.draft, a.draft_stride, a.draft_fp32, r, x), q.top, t) / q.sum;
                            stays = (double)a.u[row] * qx < px;
                        }
                    }
                }
            }
            if (lane == 0) {
                if (stays) {
                    a.out[row] = x;
                    if (a.logprobs) a.logprobs[row] = (float)lp;
                } else shared = d, kept = row - begin, done = 1;
            }
        }
        __syncthreads();
        const bool all = done != 0;
        __syncthreads();                                        // (before the first wave goes on to the next row)
        if (all) break;
    }
    const int at = begin + kept;
    Draw d = shared;
    double v = a.v[b];
    v = v > 0.0 ? v < 1.0 ? v : 1.0 : 0.0;
    int token = -1;
    if (d.from == kTop) token = d.x;
    else if (d.from != kNothing) {
        if (a.fp32) token = a.draft_fp32 ? draw_from<true, true>(d, a.V, v) : draw_from<true, false>(d, a.V, v);
        else token = a.draft_fp32 ? draw_from<false, true>(d, a.V, v) : draw_from<false, false>(d, a.V, v);
    }
    if (tid == 0) {
        a.accepted[b] = kept;
        if (a.next) a.next[b] = token;
        a.out[at] = token;
        if (a.logprobs) {
            double lp = d.from == kTop ? 0.0 : __builtin_nan("");
            if (d.from != kTop && token >= 0)
                lp = ((double)logit_at(a.logits, a.stride, a.fp32, at, token) - d.p_top) * t.c / kLog2e + log(d.p_scale);
            a.logprobs[at] = (float)lp;
        }
    }
    for (int i = at + 1 + tid; i < end; i += kVerifyThreads) {
        a.out[i] = -1;
        if (a.logprobs) a.logprobs[i] = 0.f;
    }
}

size_t carve_verify(VerifyLaunch &a, int num_cus, bool drafted, void *base)
{
    (void)num_cus;
    a.parts = 1, a.part_len = a.V;
    const size_t rows = ((size_t)a.R * a.parts * sizeof(RowPart) + 255) & ~(size_t)255;
    a.row = (RowPart *)base;
    a.draft_row = base && drafted ? (RowPart *)((char *)base + rows) : nullptr;
    return drafted ? 2 * rows : rows;
}

hipError_t launch_verify(const VerifyLaunch &a, hipStream_t s)
{
    if (a.R > 0) {
        const unsigned blocks = (unsigned)a.R * (unsigned)a.parts * (a.draft ? 2u : 1u); // (at most 2^23: R is at most 2^22, parts 1 there)
        hipLaunchKernelGGL(verify_rows_kernel, dim3(blocks), dim3(kVerifyThreads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(verify_draw_kernel, dim3((unsigned)a.B), dim3(kVerifyThreads), 0, s, a);
    return hipGetLastError();
}

} // namespace ra
