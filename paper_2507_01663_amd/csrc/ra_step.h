// Internal interface between ra_step_api.cpp and the kernels of both ends of a step (ra_pages.hip, ra_verify.hip).
#pragma once
#include "ra_internal.h"

namespace ra {

// Sequences that the kernels of the pages go over at a time, by 32-bit numbers: the first behind the last tile is one, too.
constexpr int32_t kTileSeqs = 1024, kMostPagedSeqs = INT32_MAX - kTileSeqs;

// Pages of the sequences of a batch (ra_place, ra_release).
struct PagesLaunch {
    int32_t B, T, num_pages, max_pages, num_groups;
    const int32_t *lens;         // place: tokens held; release: tokens kept
    const int32_t *asked;        // place
    const int32_t *held;
    const int32_t *group, *pfx_off, *pfx_pages;
    const int32_t *free_count;
    int32_t *stack;              // free pages; place only reads them
    int32_t *table;              // release only reads it
    int32_t *cu, *lens_out, *held_out, *free_out;
    int32_t *positions, *seqs;   // place, each may be null
    int64_t *slots;
};
hipError_t launch_place(const PagesLaunch &a, int num_cus, hipStream_t s);
hipError_t launch_release(const PagesLaunch &a, int num_cus, hipStream_t s);

// What is known of one part of a row of logits: the largest, and the sum of the weights 2^((l - largest) log2(e) / T), or for a
// greedy row the first index of the largest.
struct RowPart {
    double sum;
    float top;                   // -inf: nothing but -inf; NaN: a NaN among them
    int32_t first;
};
// A draw from p - q, or one that binary32 sums did not settle.
struct OpenDraw {
    int32_t b, from, row, x;     // from: see DrawFrom; x: the draft that was turned down
    int32_t q_row, arrived;      // row of the draft model's logits; workgroups that have added up their part
    float T, p_top, q_top;       // the rows' largest, and 1 / their sums as they are known
    double p_scale, q_scale;
};
// Sums over a part of its rows, in binary64 (see verify_left_kernel).
struct OpenPart {
    double p, q, more, under, near;
};
struct VerifyLaunch {
    int32_t B, R, V, parts, part_len; // a row's parts, and the values of a part
    int32_t fp32, draft_fp32, total_draft_rows;
    const void *logits, *draft;
    int64_t stride, draft_stride;
    const int32_t *cu, *tokens, *draft_rows;
    const float *temperature, *u, *v;
    int32_t *accepted, *out, *next;
    float *logprobs;
    RowPart *row, *draft_row;    // [R][parts]
    double *rest;                // [R][parts]  sums of what open draws are from
    int32_t *opened;             // [1]         open draws
    OpenDraw *open;              // [B]
    OpenPart *left;              // [B][parts]
    int32_t num_cus;
    int32_t alone;               // a part to a wave, not to a workgroup
    int32_t exact;               // all sums in binary64 from the start
    double eps;                  // else: what a sum may be off by, in parts of the row's
};
// How a call is divided (from B, R, V, fp32), and its workspace: the bytes; places the pointers when base is not null.
size_t carve_verify(VerifyLaunch &a, int num_cus, int64_t few, bool drafted, void *base);
bool verify_fits(int32_t B, int32_t R, int32_t V, bool drafted); // in one launch each
hipError_t launch_verify(const VerifyLaunch &a, hipStream_t s);

} // namespace ra
