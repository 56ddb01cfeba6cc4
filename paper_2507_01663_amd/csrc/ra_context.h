// The context behind the C ABI, shared by the files that implement it (ra_api.cpp, ra_chunk_api.cpp).
#pragma once
#include "../../include/rollout_attn.h"
#include "ra_internal.h"

struct ra_ctx {
    int device;
    void *scratch_ptr; // device address of `scratch` on this context's device
    int num_cus;
    int waves[2][2];  // resident attention waves, [e4m3 KV][D == 128]
    int stages[2][2]; // LDS ring depth, same indices
    int cost_prefix[2]; // scheduling weight of a shared-prefix page, [e4m3 KV]
    int cost_item;   // ... of a segment, on top of its pages
    int cost_item_pfx[2]; // ... of a shared-prefix row's segment (bf16, e4m3 pools)
    int xcd_w[8];              // default share of the page stream per accelerator die, per mille of the mean
    int32_t *wave_cum[2][2];   // device: running sums of the workgroups' shares, [e4m3 KV][D == 128], kMaxWaves + 1 each
    uint32_t *tickets;         // device: the streaming probe's ticket counter (cleared by every launch that uses it)
    int prefill_stay;          // -1: the prefill launch chooses by the batch; else ROLLOUT_ATTN_PREFILL_WGS_PER_DIE
    void *zeros;  // 256 bytes of zeros on the device
    int self_plan; // attention waves may plan their spans themselves (no schedule kernel)
    int64_t verify_few; // bf16 logits of a verification up to which all sums are binary64 (ROLLOUT_ATTN_VERIFY_FEW)
    int direct;    // batches that direct_plan says so may go without a schedule
    int32_t *host_flags; // pinned, for RA_FLAG_VALIDATE
    int timing;          // record events around the phases
    int timed;           // a decode call has recorded them (2: with a schedule launch between the first two)
    hipEvent_t ev[4];
    char err[512];
};

namespace ra {

// Text of a failure: kept in the context, or for calls without one in the thread.
__attribute__((format(printf, 2, 3))) void set_err(ra_ctx *ctx, const char *fmt, ...);

} // namespace ra
