// The launches of the attention of chunks over the paged cache (the kernels: ra_extend.h).
#include "ra_extend.h"

namespace ra {

// How many workgroups a call takes, and how finely its work is cut.
// An item of S stages that is cut in two saves half of them, and pays for a second workgroup's fixed part and for the merge, a
// kernel of its own: about 10 us.  So none is cut where the page table has room for short items only, and a workgroup takes each
// without looking at the others: up to kExShort stages beside the fixed part where there are few items, up to kExShortMany
// where there is one for every compute unit.  (Times in us uncut and cut, 28 heads on four, D = 128, bf16: one item for every
// second unit, 17 stages of few rows 19.6, 32.0, 24 21.7, 27.7, 34 27.5, 33.6, 45 33.4, 37.0; one for each, 17 stages 23.2, 38.0, 24
// 27.0, 37.0, 34 34.9, 48.8, 45 43.0, 55.5; 320 of 36 stages and more than 64 rows, e4m3, D = 64: 44.2, 41.8.)
// kExLeast: stages of a span at least, beside the fixed part.  (Eight items of 34 stages to 64 rows and 26 to 32, cut: 6 is 23.1
// and 21.3 us, 5 24.5 and 19.6, 12 32.5 and 28.5; 36 stages 23.0, 26.4, 33.0.)
constexpr int kExLeast = 6, kExShort = 20, kExShortMany = 36;
static void extend_shape(ExtendLaunch &a)
{
    const int64_t rows = (int64_t)a.max_chunk * a.G; // of a kv head, at most
    a.few = rows <= kExRows;
    // Many sequences far shorter than the longest: the short ones apart.  (64 sequences, 62, 56, 48, 32 of them single tokens, the
    // others of 200, 32 heads on eight, e4m3: 55.0, 84.8, 143, 223 us, in one line 76.0, 107, 143, 223; bf16 80.5, 94.5, 120, 192, in one
    // line 77.5, 98.8, 121, 193.)
    a.two = rows > 64 && 4 * (int64_t)a.T <= (int64_t)a.B * a.max_chunk;
    const int64_t blocks = a.few ? a.B : (int64_t)a.T * a.G / kExRows + a.B, items = blocks * a.Hkv;
    const int most = rows <= 64 ? (int)rows : 65, fixed = ex_fixed(most, a.two), longest = fixed + 1 + ex_weight(a.max_pages / 2 + 1, most); // an item at most
    a.least = kExLeast + fixed;
    a.direct = longest <= (items < a.num_cus ? kExShort : kExShortMany) + fixed;
    const int64_t resident = (int64_t)(a.num_cus < 8 ? 8 : a.num_cus & ~7) * (a.D == 64 ? 3 : 2);
    int64_t spans = (items * longest / a.least + 7) & ~(int64_t)7;
    spans = spans < 16 ? 16 : spans < resident ? spans : resident; // (two lines take eight each, at least)
    a.spans = (int)(spans < kExMaxSpans ? spans : kExMaxSpans);
    // (a workgroup for every item where items are left whole, or may be: see ex_walk, and ExLine::measure)
    const int gg_shift = (a.Hkv & 7) == 0 ? 3 : (a.Hkv & 3) == 0 ? 2 : (a.Hkv & 1) == 0 ? 1 : 0, s_shift = 3 - gg_shift;
    const int64_t each = 8 * ((blocks * (a.Hkv >> gg_shift) + (1 << s_shift) - 1) >> s_shift);
    a.grid = (int)(a.direct || items >= 2 * a.spans ? each : a.spans);
}

size_t carve_extend(ExtendLaunch &a, void *base)
{
    extend_shape(a);
    if (a.direct) return 0;
    const int64_t slots = 2 * (int64_t)a.spans, rows = kExRows;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        void *const p = base ? (char *)base + at : nullptr;
        at += (bytes + 255) & ~(size_t)255;
        return p;
    };
    a.desc = (int4 *)take(sizeof(int4) * 2 * a.spans);
    a.part_lse = (float *)take((size_t)(slots * rows * 8));
    a.part_o = (float *)take((size_t)(slots * rows * a.D * 4));
    return at;
}

#define RA_EX_KINDS(X, DD, F) X(DD, F, kExAny) X(DD, F, kEx32) X(DD, F, kEx64) X(DD, F, kExTwo)
#define RA_EX_KERNELS(X) RA_EX_KINDS(X, 64, false) RA_EX_KINDS(X, 64, true) RA_EX_KINDS(X, 128, false) RA_EX_KINDS(X, 128, true)

hipError_t extend_config()
{
    hipError_t e = hipSuccess;
#define RA_EX_CONFIG(DD, F, K) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)extend_kernel<DD, F, K>, hipFuncAttributeMaxDynamicSharedMemorySize, (ExTileLds<DD, F>::kBytes));
    RA_EX_KERNELS(RA_EX_CONFIG)
#undef RA_EX_CONFIG
    return e;
}

hipError_t launch_extend(const ExtendLaunch &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.grid), block(64 * kExWaves);
    const int64_t rows = (int64_t)a.max_chunk * a.G;
    const ExKind kind = rows <= 32 ? kEx32 : rows <= 64 ? kEx64 : a.two ? kExTwo : kExAny;
#define RA_EX_LAUNCH(DD, F, K) \
    if (a.D == DD && (a.kv_fp8 != 0) == F && kind == K) hipLaunchKernelGGL((extend_kernel<DD, F, K>), grid, block, (ExTileLds<DD, F>::kBytes), s, EX_GIVE(a));
    RA_EX_KERNELS(RA_EX_LAUNCH)
#undef RA_EX_LAUNCH
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.direct) return e;
    if (a.D == 128) hipLaunchKernelGGL(extend_merge_kernel<128>, dim3((unsigned)(kExMergeWgs * a.spans)), block, 0, s, a.desc, a);
    else hipLaunchKernelGGL(extend_merge_kernel<64>, dim3((unsigned)(kExMergeWgs * a.spans)), block, 0, s, a.desc, a);
    return hipGetLastError();
}

} // namespace ra
