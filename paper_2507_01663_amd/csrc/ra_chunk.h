// Internal interface between ra_chunk_api.cpp and the kernels for chunks of new tokens (ra_rotate.hip, ra_extend.hip).
#pragma once
#include "ra_internal.h"

namespace ra {

// Norm, rotation and append (ra_rotate, ra_append_chunk): element (t, head, d) of a tensor lies at t * stride + head * D + d.
struct RowsLaunch {
    int32_t T, Hq, Hkv, D;       // Hq or Hkv 0: that tensor is not touched
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;     // k_out: without a cache
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    const float *qw, *kw;        // null: no norm
    float eps;
    const int32_t *positions;    // null with a cache: the position in the sequence
    const float *rope;           // [rope_len][rot]
    int32_t rope_len, rot, interleaved;
    int32_t slots_shift;         // row slots of a token in a wave's pass (set by launch_rows)
    // the cache
    int32_t B, max_chunk, max_pages, num_pages;
    const int32_t *cu, *seq_lens, *table;
    uint8_t *k_pool, *v_pool;
    int64_t stride_page_b, stride_head_b; // bytes
    int32_t stride_token_b;
    float *k_scale, *v_scale;    // e4m3 pools
};
hipError_t launch_rotate(const RowsLaunch &a, int num_cus, hipStream_t s);
hipError_t launch_append_chunk(const RowsLaunch &a, int kv_fp8, int num_cus, hipStream_t s);

// Attention of chunks over the cache (ra_extend).
struct ExtendLaunch {
    int32_t B, T, max_chunk, Hq, Hkv, D, G;
    int32_t num_pages, max_pages, kv_fp8, num_cus;
    uint32_t magic_g;            // ceil(2^32 / G)
    const uint16_t *q;
    int64_t q_stride;            // elements
    const int32_t *cu, *seq_lens, *table;
    const uint8_t *k_pool, *v_pool;
    int64_t stride_page_b, stride_head_b; // bytes
    int32_t stride_token_b;
    const float *k_scale, *v_scale;
    float scale_log2;            // softmax_scale * log2(e)
    uint16_t *out;
    float *lse;
    const void *zeros;
    float *part_o, *part_lse;    // partial results, two slots per span
    int4 *desc;                  // [spans][2] what the merge adds up
    // (set by carve_extend) workgroups that share the work, workgroups launched, length of a span at least, whether every
    // sequence is one block, whether no item is long enough to be cut, and whether short sequences have a line of their own
    int32_t spans, grid, least, few, direct, two;
};
// How a call is launched (from B, T, max_chunk, Hkv, G, D, max_pages and num_cus), and its workspace: the bytes; places the pointers
// when base is not null.
size_t carve_extend(ExtendLaunch &a, void *base);
hipError_t extend_config();
hipError_t launch_extend(const ExtendLaunch &a, hipStream_t s);

} // namespace ra
