// What the verification's kernels read of a row, run on the host: the kernels' own functions, with arrays that end at a page that no one may
// read.  A read past an array's documented end, or of one that is documented not to be read, ends the program by a signal.
// Prints one line for each thing that it has looked at.
#include <hip/hip_runtime.h>
#include <sys/mman.h>

#include <cstdio>
#include <cstdlib>

#include "ra_device.h"
#include "ra_internal.h"

// The functions are for the host, too, and there are no kernels.
__host__ static inline float __uint_as_float(unsigned x) { return __builtin_bit_cast(float, x); }
#undef __global__
#define __global__ inline
#undef __launch_bounds__
#define __launch_bounds__(...)
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(...) ((void)0)
#pragma clang force_cuda_host_device begin
#include "ra_verify.hip"
#pragma clang force_cuda_host_device end

// n elements whose end is the end of what may be read.
template <typename T> static T *ending(size_t n)
{
    constexpr size_t kPages = 16 * 4096;
    char *const m = (char *)mmap(nullptr, 2 * kPages, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (m == MAP_FAILED || mprotect(m + kPages, kPages, PROT_NONE)) abort();
    return (T *)(m + kPages) - n;
}

static void done(const char *what)
{
    puts(what);
    fflush(stdout);
}

int main()
{
    using namespace ra;
    constexpr int R = 5, V = 40;
    VerifyLaunch a = {};
    a.B = 2, a.R = R, a.V = V, a.parts = 1, a.part_len = 4096, a.fp32 = 1, a.stride = V;
    int32_t *const cu = ending<int32_t>(3), *const tokens = ending<int32_t>(R), *const draft_rows = ending<int32_t>(2);
    float *const logits = ending<float>(R * V);
    cu[0] = 0, cu[1] = 2, cu[2] = R;
    for (int t = 0; t < R; t++) tokens[t] = t + 3;
    for (int i = 0; i < R * V; i++) logits[i] = 0.01f * i;
    a.cu = cu, a.tokens = tokens, a.logits = logits;
    a.row = ending<RowPart>(R);

    // the last row of the batch has no number of its own to be accepted by
    float *const u = ending<float>(R - 1);
    for (int t = 0; t < R - 1; t++) u[t] = 0.1f * t;
    a.u = u;
    for (int t = 0; t < R; t++) {
        const Early e = ask_early(a, t, 0);
        if (e.row != t || (t < R - 1 && (e.x != t + 4 || e.u != u[t]))) return 1;
    }
    done("numbers");

    // a greedy sequence's drafts are judged without the draft model's logits: there may be none at their address
    draft_rows[0] = 0, draft_rows[1] = 1;
    a.draft = ending<float>(0), a.draft_rows = draft_rows, a.draft_stride = V, a.draft_fp32 = 1, a.total_draft_rows = 3, a.draft_row = ending<RowPart>(R);
    for (int b = 0; b < 2; b++)
        for (int t = cu[b]; t < cu[b + 1]; t++) {
            const Asked r = ask_row(a, b, ask_early(a, t, 0), cu[b + 1], temper_from(0.f));
            if (r.row != t || r.q_row >= 0 || r.x != (t + 1 < cu[b + 1] ? t + 4 : -1) || (r.x >= 0 && r.l != logits[t * V + r.x])) return 2;
        }
    done("greedy");

    // others are judged with them
    float *const draft = ending<float>(3 * V);
    for (int i = 0; i < 3 * V; i++) draft[i] = -0.5f * i;
    a.draft = draft;
    for (int b = 0; b < 2; b++)
        for (int t = cu[b]; t < cu[b + 1] - 1; t++) {
            const Asked r = ask_row(a, b, ask_early(a, t, 0), cu[b + 1], temper_from(1.f));
            if (r.q_row != draft_rows[b] + t - cu[b] || r.m != draft[r.q_row * V + r.x]) return 3;
        }
    done("drafts");
    return 0;
}
