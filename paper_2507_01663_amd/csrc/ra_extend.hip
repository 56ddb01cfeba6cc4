// The launches of the attention of chunks over the paged cache (the kernels: ra_extend.h).
#include "ra_extend.h"

namespace ra {

// Which kernel a call takes, its workgroups, and how finely the work is cut.
// An item of S stages that is cut in two saves half of them, and pays for a second workgroup's fixed part and the merge, a
// kernel of its own: kExCut.
constexpr int kExLeast = 10, kExLeastFew = 16, kExCut = 20, kExCutFew = 32;
static void extend_shape(ExtendLaunch &a)
{
    a.few = (int64_t)a.max_chunk * a.G <= kExFewRows;
    const int64_t blocks = a.few ? a.B : (int64_t)a.T * a.G / kExTileRows + a.B, items = blocks * a.Hkv;
    const int longest = a.max_pages / 2 + 1 + (a.few ? kExFixed<kExFewRows> : kExFixed<kExTileRows>); // an item at most
    a.least = a.few ? kExLeastFew : kExLeast;
    a.cut = a.few ? kExCutFew : kExCut;
    a.direct = longest <= a.cut;
    const int64_t resident = (int64_t)(a.num_cus < 8 ? 8 : a.num_cus & ~7) * (a.few ? (a.D == 64 ? 2 : 1) : (a.D == 64 ? 3 : 2));
    int64_t spans = (items * longest / a.least + 7) & ~(int64_t)7;
    spans = spans < 8 ? 8 : spans < resident ? spans : resident;
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
    const int64_t slots = 2 * (int64_t)a.spans, rows = a.few ? kExFewRows : kExTileRows;
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

#define RA_EX_TILES(X) X(64, false) X(64, true) X(128, false) X(128, true)
#define RA_EX_FEWS(X) X(64, 2, 1) X(64, 2, 2) X(64, 1, 1) X(64, 1, 2) X(128, 2, 1) X(128, 2, 2) X(128, 1, 1) X(128, 1, 2)

hipError_t extend_config()
{
    hipError_t e = hipSuccess;
#define RA_EX_CONFIG(DD, F) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)extend_tile_kernel<DD, F>, hipFuncAttributeMaxDynamicSharedMemorySize, (ExTileLds<DD, F>::kBytes));
    RA_EX_TILES(RA_EX_CONFIG)
#undef RA_EX_CONFIG
#define RA_EX_CONFIG(DD, KVB, Q) \
    if (e == hipSuccess) e = hipFuncSetAttribute((const void *)extend_few_kernel<DD, KVB, Q>, hipFuncAttributeMaxDynamicSharedMemorySize, ExFewLds<DD, KVB>::kBytes);
    RA_EX_FEWS(RA_EX_CONFIG)
#undef RA_EX_CONFIG
    return e;
}

hipError_t launch_extend(const ExtendLaunch &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.grid), block(64 * kExWaves);
    if (!a.few) {
#define RA_EX_LAUNCH(DD, F) \
    if (a.D == DD && (a.kv_fp8 != 0) == F) hipLaunchKernelGGL((extend_tile_kernel<DD, F>), grid, block, (ExTileLds<DD, F>::kBytes), s, EX_GIVE(a));
        RA_EX_TILES(RA_EX_LAUNCH)
#undef RA_EX_LAUNCH
    } else {
        const int rows = a.max_chunk * a.G, tiles = rows <= 16 ? 1 : 2;
#define RA_EX_LAUNCH(DD, KVB, Q) \
    if (a.D == DD && (a.kv_fp8 ? 1 : 2) == KVB && tiles == Q) hipLaunchKernelGGL((extend_few_kernel<DD, KVB, Q>), grid, block, (ExFewLds<DD, KVB>::kBytes), s, EX_GIVE(a));
        RA_EX_FEWS(RA_EX_LAUNCH)
#undef RA_EX_LAUNCH
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.direct) return e;
#define RA_EX_MERGE(DD) \
    if (a.few) hipLaunchKernelGGL((extend_merge_kernel<DD, kExFewRows>), dim3(kExMergeWgs), block, 0, s, a.desc, a.spans, a); \
    else hipLaunchKernelGGL((extend_merge_kernel<DD, kExTileRows>), dim3(kExMergeWgs), block, 0, s, a.desc, a.spans, a)
    if (a.D == 128) {
        RA_EX_MERGE(128);
    } else {
        RA_EX_MERGE(64);
    }
#undef RA_EX_MERGE
    return hipGetLastError();
}

} // namespace ra
