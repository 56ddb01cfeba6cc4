// gfx950 kernels of the pages of a batch: places of new tokens (block table, packed offsets, positions, slots) and pages back to
// the stack of free ones.
//
// Integers only.  A sequence's share of the stack and of the packed arrays is a running sum over the sequences before it, so a
// workgroup goes over all sequences, 1024 at a time with one to a thread, and then over the tokens (or the pages) of that tile: each
// finds its sequence by bisection of the tile's running sums in LDS.  A page of the stack that a sequence takes begins at one of its
// new tokens, so the token that begins a page also writes it into the table.
//
// Trips to memory bound them: lengths (and a group's offsets behind them), the page, the store.  So there is one kernel where it can be
// (a second costs 3 us), every workgroup makes all sums itself instead of waiting for another's, and a step's few tokens are placed by
// the threads that have their sequences, without the search.  Measured: 256 sequences of one token 4.2 us (a launch), 777 turns of which
// the last find no pages 5.9 (the sums are made twice), 495 000 tokens of 512 prompts 6.5, of which 8 MB of stores would take 1.6; 1.2
// million pages of 2 048 sequences back 7.3.  A tile of 1024 sequences begins when the one before is done: 2 000 sequences of one token 10.6, 4 000
// 17.5; back 4.7 and 7.2.
#include "ra_device.h"
#include "ra_step.h"
#include "ra_wave.h"

namespace ra {

constexpr int kTileWaves = kTileSeqs / 64;

// Inclusive sums over the 1024 threads of a workgroup, on top of what was carried in; the new totals are carried out.  (Tokens of sequences
// that a table has room for are fewer than 2^35: whole numbers of binary64.)
struct TwoSums {
    int32_t pages;
    double tokens;
};
struct ScanLds {
    int32_t pages[kTileWaves];
    double tokens[kTileWaves];
};
__device__ __forceinline__ TwoSums scan(TwoSums x, TwoSums &carry, ScanLds &lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    x.pages = wave_scan(x.pages), x.tokens = wave_scan(x.tokens);
    if (lane == 63) lds.pages[wave] = x.pages, lds.tokens[wave] = x.tokens;
    __syncthreads();
    TwoSums all = carry;
#pragma unroll
    for (int w = 0; w < kTileWaves; w++) {
        if (w == wave) x.pages += all.pages, x.tokens += all.tokens;
        all.pages += lds.pages[w], all.tokens += lds.tokens[w];
    }
    carry = all;
    return x;
}

// Pages that sequence b's group shares, and where they are listed.
__device__ __forceinline__ int shared_pages(const PagesLaunch &a, int b, int &at)
{
    at = 0;
    if (a.num_groups <= 0) return 0;
    const int g = a.group[b];
    if (g < 0 || g >= a.num_groups) return 0;
    at = a.pfx_off[g];
    const int n = a.pfx_off[g + 1] - at;
    return n > 0 && at >= 0 ? n : 0;
}

__device__ __forceinline__ int stack_height(const PagesLaunch &a)
{
    const int n = a.free_count[0];
    return n < 0 ? 0 : n > a.num_pages ? a.num_pages : n;
}

// The last of the tile's sequences whose sum of those before it is at most x (a sequence without any has the sum of the next).
__device__ __forceinline__ int owner(const int32_t *before, int x)
{
    int lo = 0;
#pragma unroll
    for (int step = kTileSeqs / 2; step > 0; step /= 2)
        if (before[lo + step] <= x) lo += step;
    return lo;
}

// This workgroup's first block of 1024 from the one that x is in: workgroup w of n has those whose number is w more than a multiple of n.
__device__ __forceinline__ int64_t first_block(int x)
{
    const unsigned n = gridDim.x, b = (unsigned)x / kTileSeqs, mine = b % n;
    return (int64_t)b + (blockIdx.x >= mine ? blockIdx.x - mine : blockIdx.x + n - mine);
}

constexpr int kOwn = 4; // a sequence with so few new tokens places them itself, where all of a tile have no more

// TOKENS: the tokens are placed, by workgroups that share the tokens in blocks of 1024; STATE: the first workgroup writes the
// new lengths, counts and offsets.  Both at once with one workgroup alone, or where no other reads what that writes.
template <bool TOKENS, bool STATE> __global__ __launch_bounds__(kTileSeqs) void place_kernel(PagesLaunch a)
{
    touch_lines(a);
    __shared__ ScanLds sums[2];
    __shared__ int32_t first[kTileSeqs];                        // tokens before the sequence
    __shared__ int4 row[kTileSeqs];                             // {tokens held, pages held, pages with the group's, stack's entry of the first taken}
    __shared__ int32_t listed[kTileSeqs];                       // where its group's pages are
    const int tid = threadIdx.x, free = stack_height(a);
    TwoSums wanted = {0, 0.0}, given = {0, 0.0};
    auto put = [&](int64_t b, int place, const int4 &r, int at, int t) {
        const int i = place / kPage;
        int32_t *const entries = a.table + b * a.max_pages;
        int page;
        if (i < r.y) page = entries[i];
        else if (i < r.z) page = a.pfx_pages[at + i];
        else {
            page = a.stack[r.w - (i - r.z)];
            if (place % kPage == 0) entries[i] = page;
        }
        if (a.positions) a.positions[t] = place;
        if (a.slots) a.slots[t] = (int64_t)page * kPage + place % kPage;
        if (a.seqs) a.seqs[t] = (int32_t)b;
    };
    for (int base = 0; base < a.B; base += kTileSeqs) {
        const int b = base + tid;
        int L = 0, n = 0, H = 0, F = 0, at = 0;
        if (b < a.B) L = a.lens[b], n = a.asked[b], H = a.held[b], F = shared_pages(a, b, at);
        const int S = H > F ? H : F;
        const int64_t end = (int64_t)L + n;
        const int64_t P = (end + kPage - 1) / kPage;
        const bool fine = n > 0 && L >= 0 && H >= 0 && S <= a.max_pages && P <= a.max_pages && L <= (int64_t)kPage * S;
        const TwoSums was = given;
        TwoSums mine = {0, 0.0};
        if (fine) mine = {P > S ? (int32_t)P - S : 0, (double)n};
        const TwoSums upto = scan(mine, wanted, sums[0]);
        const bool served = fine && (mine.pages == 0 || upto.pages <= free) && upto.tokens <= a.T;
        TwoSums incl = upto;
        if (wanted.pages > free || wanted.tokens > a.T) {       // (else all are served, so far, and these are the sums)
            if (!served) mine = {0, 0.0};
            incl = scan(mine, given, sums[1]);
        } else given = wanted;
        const int32_t cu = (int32_t)(incl.tokens - mine.tokens);
        if (STATE && b < a.B && blockIdx.x == 0) {
            a.cu[b] = cu;
            a.lens_out[b] = served ? L + n : L;
            a.held_out[b] = served && P > S ? (int32_t)P : served ? S : H;
        }
        if (TOKENS) {
            const int4 r = make_int4(L, H, S, free - 1 - (incl.pages - mine.pages));
            const int t0 = (int)was.tokens, t1 = (int)given.tokens;
            if (served && F > H && (cu / kTileSeqs) % gridDim.x == blockIdx.x)
                for (int i = H; i < F; i++) a.table[(int64_t)b * a.max_pages + i] = a.pfx_pages[at + i];
            if (t1 - t0 <= kTileSeqs && gridDim.x == 1 && __syncthreads_and(n <= kOwn || !served)) {
                for (int i = 0; served && i < n; i++) put(b, L + i, r, at, cu + i);
                continue;
            }
            first[tid] = cu, row[tid] = r, listed[tid] = at;
            __syncthreads();
            for (int64_t blk = first_block(t0); blk * kTileSeqs < t1; blk += gridDim.x) {
                const int64_t t = blk * kTileSeqs + tid;
                if (t < t0 || t >= t1) continue;
                const int s = owner(first, (int)t);
                put(base + s, row[s].x + (int)t - first[s], row[s], listed[s], (int)t);
            }
        }
        if (base + kTileSeqs < a.B) __syncthreads();
    }
    if (TOKENS && (a.positions || a.slots || a.seqs))
        for (int64_t t = (int64_t)given.tokens + (int64_t)blockIdx.x * kTileSeqs + tid; t < a.T; t += (int64_t)gridDim.x * kTileSeqs) {
            if (a.positions) a.positions[t] = -1;
            if (a.slots) a.slots[t] = -1;
            if (a.seqs) a.seqs[t] = -1;
        }
    if (STATE && tid == 0 && blockIdx.x == 0) a.cu[a.B] = (int32_t)given.tokens, a.free_out[0] = free - given.pages;
}

template <bool PAGES, bool STATE> __global__ __launch_bounds__(kTileSeqs) void release_kernel(PagesLaunch a)
{
    touch_lines(a);
    __shared__ ScanLds sums;
    __shared__ int32_t first[kTileSeqs], begin[kTileSeqs];      // pages before the sequence's, and its first that goes back
    const int tid = threadIdx.x, free = stack_height(a);
    TwoSums back = {0, 0.0};
    for (int base = 0; base < a.B; base += kTileSeqs) {
        const int b = base + tid, before = back.pages;
        int keep = 0, H = 0, F = 0, at;
        if (b < a.B) keep = a.lens[b], H = a.held[b], F = shared_pages(a, b, at);
        const int kept = keep > 0 ? (int)(((int64_t)keep + kPage - 1) / kPage) : 0, K = kept < H ? kept : H;
        const bool fine = H >= 0 && H <= a.max_pages;
        const int from = K > F ? K : F;
        const TwoSums mine = {fine && from < H ? H - from : 0, 0.0};
        const TwoSums incl = scan(mine, back, sums);
        if (STATE && b < a.B && blockIdx.x == 0) a.held_out[b] = fine ? K : H;
        if (PAGES) {
            first[tid] = incl.pages - mine.pages, begin[tid] = from;
            __syncthreads();
            for (int64_t blk = first_block(before); blk * kTileSeqs < back.pages; blk += gridDim.x) {
                const int64_t at64 = blk * kTileSeqs + tid;
                if (at64 < before || at64 >= back.pages) continue;
                const int e = (int)at64;
                const int s = owner(first, e);
                const int64_t to = (int64_t)free + e;
                if (to < a.num_pages) a.stack[to] = a.table[(int64_t)(base + s) * a.max_pages + begin[s] + e - first[s]];
            }
        }
        if (base + kTileSeqs < a.B) __syncthreads();
    }
    if (STATE && tid == 0 && blockIdx.x == 0) a.free_out[0] = (int64_t)free + back.pages < a.num_pages ? free + back.pages : a.num_pages;
}

// Workgroups that share n tokens (or pages): one up to kAlone of them, else one for each 1024.  The first writes the state too, unless it is
// written where the others still read it: then a kernel of its own does.
constexpr int kAlone = 4096;
static unsigned workgroups(int64_t n, int num_cus)
{
    const int64_t w = (n + kTileSeqs - 1) / kTileSeqs;
    return n <= kAlone ? 1u : w < num_cus ? (unsigned)w : (unsigned)num_cus;
}

hipError_t launch_place(const PagesLaunch &a, int num_cus, hipStream_t s)
{
    const dim3 n(workgroups(a.T, num_cus)), threads(kTileSeqs);
    if (n.x == 1 || (a.lens_out != a.lens && a.held_out != a.held && a.free_out != a.free_count)) {
        hipLaunchKernelGGL((place_kernel<true, true>), n, threads, 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((place_kernel<true, false>), n, threads, 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((place_kernel<false, true>), dim3(1), threads, 0, s, a);
    return hipGetLastError();
}

hipError_t launch_release(const PagesLaunch &a, int num_cus, hipStream_t s)
{
    const dim3 n(workgroups((int64_t)a.B * a.max_pages, num_cus)), threads(kTileSeqs);
    if (n.x == 1 || (a.held_out != a.held && a.free_out != a.free_count)) {
        hipLaunchKernelGGL((release_kernel<true, true>), n, threads, 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((release_kernel<true, false>), n, threads, 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((release_kernel<false, true>), dim3(1), threads, 0, s, a);
    return hipGetLastError();
}

} // namespace ra
