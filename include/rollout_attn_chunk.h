/*
 * rollout_attn, chunks of new tokens: the layer of a step that puts more than
 * one token, or a first token, into sequences that already have a paged cache.
 *
 * Setting.  Between a prompt's prefill and single decode steps (rollout_attn.h)
 * a rollout worker meets chunks: the tokens of a tool's output or of a user's
 * turn go into every response of a multi-turn rollout, a long prompt is taken in
 * pieces between decode steps, a draft of a few tokens is checked at once.  A
 * layer of such a step is, after its projection of queries, keys and values:
 *   rollout_attn_append_chunk   norms and rotates the chunk's queries and keys by
 *                               head and writes keys and values into the pages;
 *   rollout_attn_extend         lets every new token attend to its sequence's
 *                               pages, the chunk's own included.
 * rollout_attn_rotate is the norm and rotation alone, for tokens that are not
 * (yet) cached: the rows that rollout_attn_prefill takes.  The paper leaves all
 * of this to its inference engine (Sec. 2.1.1); this header defines it.
 *
 * Contexts, streams, ownership of memory, status codes and error texts are
 * those of rollout_attn.h: no call allocates, copies or waits, each enqueues
 * kernels on the given stream and nothing else, and so may be recorded into a HIP
 * graph; inputs may be reused or freed once the stream has passed the call.
 * Results are deterministic: the same inputs give the same bytes.
 */
#ifndef ROLLOUT_ATTN_CHUNK_H
#define ROLLOUT_ATTN_CHUNK_H

#include "rollout_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Norm and rotation of query and key rows by head.  For row x (D values) of one head of token t, in IEEE binary32
 * and rounded once, to bf16, at the end:
 *   norm      y = x * w / sqrt(mean_d(x_d^2) + eps)          (weight given; else y = x)
 *   rotation  for j < rot_dim / 2, with c, s = rope[p][j], rope[p][rot_dim / 2 + j], p = positions[t]:
 *               (y_a, y_b) -> (y_a c - y_b s, y_b c + y_a s)
 *             a, b = j, j + rot_dim / 2, or 2 j, 2 j + 1 when interleaved != 0; d >= rot_dim stay as they are.
 * Layout: element (t, head, d) of a tensor at t * stride_token + head * D + d, so that the three parts of one
 * projection's output can be given as they lie.  Strides in elements, multiples of 8 and at least heads * D; pointers
 * 16-byte aligned, q_weight and k_weight too.  q and q_out (k and k_out) may be the same memory with the same stride;
 * otherwise outputs overlap nothing.  q == NULL or k == NULL: that tensor is not touched.
 * A token whose position is not in [0, rope_len) is left out: its rows of q_out and k_out keep what they hold.
 * Supported: D in {64, 128}; rot_dim a multiple of 16, 0 .. D (0: no rotation; rope and positions are not read).
 */
typedef struct {
    int32_t num_tokens, Hq, Hkv, D;
    const void *q;             /* dev, bf16, or NULL */
    const void *k;             /* dev, bf16, or NULL */
    void *q_out;               /* dev, bf16 */
    void *k_out;               /* dev, bf16 */
    int64_t q_stride_token, k_stride_token, q_out_stride_token, k_out_stride_token;
    const float *q_weight;     /* dev fp32 [D], or NULL: the queries are not normalised */
    const float *k_weight;     /* dev fp32 [D], or NULL: nor are the keys */
    float eps;                 /* >= 0; read where a weight is given */
    const int32_t *positions;  /* dev [num_tokens] */
    const float *rope;         /* dev fp32 [rope_len][rot_dim], 16-byte aligned */
    int32_t rope_len, rot_dim, interleaved;
} ra_rotate;

/* Host-only check of the scalars, strides and pointers (device data is not read): what rollout_attn_rotate would return
 * for them before touching the device.  msg (may be NULL) receives a NUL-terminated explanation. */
ra_status rollout_attn_check_rotate(const ra_rotate *rotate, char *msg, size_t msg_len);

/* Enqueues the norm and rotation: one kernel. */
ra_status rollout_attn_rotate(ra_ctx *ctx, const ra_rotate *rotate, void *hip_stream);

/*
 * Append of a chunk of new tokens per sequence to the paged cache.  Sequence b's new tokens are the packed tokens
 * [cu_seqlens[b], cu_seqlens[b+1]); token i of them goes to position p = seq_lens[b] + i, seq_lens[b] being the length
 * BEFORE the append (it is not modified): page block_table[b][p / page_size], slot p % page_size, every kv head, of pools
 * laid out as in ra_problem.
 *   keys      rot.k, normalised and rotated as rollout_attn_rotate does it, with positions[t] or, when rot.positions is
 *             NULL, with p; rot.k_weight == NULL and rot.rot_dim == 0: as they are
 *   values    v, as they are (laid out like rot.k)
 *   queries   rot.q, if not NULL: normalised and rotated into rot.q_out beside them
 * rot.num_tokens is the chunk's total, cu_seqlens[num_seqs]; rot.k_out must be NULL; rot.q_out may be rot.q as for rollout_attn_rotate.
 *   bf16 pools: keys are rounded to bf16, once, from binary32.
 *   e4m3 pools, per (page, kv head), K and V alike, in binary32 with round-to-nearest-even, a = largest |x| among the new
 *   rows of the page (a NaN does not take part):
 *     the page's first slot is among the new ones: scale = a > 0 ? a / 448 : 1;
 *     else: if a <= scale * 448 the page keeps its scale, else scale' = a / 448 and the slots before the new ones are
 *       re-quantised, code = enc((dec(code) * scale) / scale');
 *     the new rows are stored as enc(x / scale); slots past them are left as they were.
 *   One token per sequence, without norm and rotation, gives the bytes that rollout_attn_append gives.
 * cu_seqlens: dev int32 [num_seqs + 1], starts at 0, non-decreasing.  max_chunk_len is a HOST-side upper bound of every
 * chunk's length; a chunk's tokens at or past it may be left out.  No two sequences may append into the same page.  Left
 * out are also: a token whose rotation position is not in [0, rope_len) (query, key and value), and the keys and values
 * of a sequence whose length is negative, that have no room in the table row (p >= max_pages_per_seq * page_size), or whose
 * page id is not in [0, num_pages).
 * Supported: page_size == 16; D in {64, 128}; otherwise as ra_rotate.
 */
typedef struct {
    ra_rotate rot;
    const void *v;             /* dev, bf16 */
    int64_t v_stride_token;
    int32_t num_seqs, max_chunk_len;
    const int32_t *cu_seqlens; /* dev */
    const int32_t *seq_lens;   /* dev [num_seqs] */
    int32_t page_size, num_pages, max_pages_per_seq;
    const int32_t *block_table; /* dev [num_seqs][max_pages_per_seq] */
    void *k_pool;              /* dev */
    void *v_pool;              /* dev */
    int64_t kv_stride_page, kv_stride_head, kv_stride_token; /* in elements */
    int32_t kv_dtype;          /* ra_kv_dtype */
    float *k_scale;            /* dev fp32 [num_pages][Hkv]; NULL unless fp8 */
    float *v_scale;
} ra_append_chunk;

ra_status rollout_attn_check_append_chunk(const ra_append_chunk *append, char *msg, size_t msg_len);

/* Enqueues the append: one kernel. */
ra_status rollout_attn_append_chunk(ra_ctx *ctx, const ra_append_chunk *append, void *hip_stream);

/*
 * Attention of a chunk of new tokens per sequence over the paged cache.  Sequence b has n = cu_seqlens[b+1] -
 * cu_seqlens[b] new tokens, L = seq_lens[b] tokens in all, the new ones last and already in the cache (seq_lens is the
 * length AFTER the append, as for rollout_attn_decode).  For its new token i, query head h, kv = h / (Hq / Hkv), k_j and
 * v_j stored as in ra_problem:
 *   s_j      = softmax_scale * <q[cu_seqlens[b] + i, h, :], k_j>,  0 <= j <= L - n + i
 *   out[.,h] = sum_j softmax(s)_j * v_j          (bf16)
 *   lse[.,h] = ln sum_j exp(s_j)                 (fp32, natural log)
 * A token that sees no key (L - n + i < 0) gives out = 0 and lse = -inf.  What a token does not see has no part in its
 * result, whatever it holds: keys and values of later tokens, slots at or past L (either may be infinite or NaN; an e4m3
 * page's scale is a part of every value in the page, and of a page without a token that is seen it has none).  seq_lens
 * outside [0, max_pages_per_seq * page_size] count as the nearest of the two; block-table entries at or past
 * ceil(L / page_size) are not read, the others must be in [0, num_pages).
 * Layout: q bf16, element (t, head, d) at t * q_stride_token + head * D + d; out bf16 [T][Hq][D] and lse fp32 [T][Hq]
 * contiguous, T = total_tokens = cu_seqlens[num_seqs].  cu_seqlens as for ra_append_chunk.  max_chunk_len is a HOST-side
 * upper bound of every chunk's length (the launch is sized by it and by total_tokens; a chunk's tokens at or past it may
 * be left unprocessed, those before it are what they are in the whole chunk).
 * One new token for every sequence (max_chunk_len == 1 and total_tokens == num_seqs) is a decode step, and runs as one
 * without a prompt-group hint where rollout_attn_decode supports the shape and q is contiguous.  Of such a call the bound
 * must hold: cu_seqlens is not read, and token b is sequence b's.
 * Supported: page_size == 16; D in {64, 128}; Hq % Hkv == 0; Hq / Hkv <= 128.
 */
typedef struct {
    int32_t num_seqs, total_tokens, max_chunk_len;
    int32_t Hq, Hkv, D;
    const void *q;             /* dev */
    int64_t q_stride_token;
    const int32_t *cu_seqlens; /* dev */
    const int32_t *seq_lens;   /* dev [num_seqs] */
    int32_t page_size, num_pages, max_pages_per_seq;
    const int32_t *block_table; /* dev [num_seqs][max_pages_per_seq] */
    const void *k_pool;        /* dev */
    const void *v_pool;        /* dev */
    int64_t kv_stride_page, kv_stride_head, kv_stride_token; /* in elements */
    int32_t kv_dtype;          /* ra_kv_dtype */
    const float *k_scale;      /* dev fp32 [num_pages][Hkv]; NULL unless fp8 */
    const float *v_scale;
    float softmax_scale;       /* positive */
    void *out;                 /* dev */
    float *lse;                /* dev */
} ra_extend;

ra_status rollout_attn_check_extend(const ra_extend *extend, char *msg, size_t msg_len);

/* Bytes of device workspace rollout_attn_extend needs for this shape (only the dimensions, the
 * page counts and kv_dtype are read).  ctx may be NULL: the
 * size for a 256-compute-unit device is returned.  0 (a batch of short sequences): none, and it may be NULL. */
ra_status rollout_attn_extend_workspace_size(const ra_ctx *ctx, const ra_extend *shape_only, size_t *bytes);

/* Enqueues the attention on hip_stream: one kernel, and a second where workgroups may share a sequence's work (a workspace size
 * other than 0); a decode step's where it runs as one.  workspace as for rollout_attn_decode: dev memory of at
 * least rollout_attn_extend_workspace_size() bytes, 256-byte aligned, contents irrelevant on entry and undefined
 * afterwards; calls that overlap in time need distinct workspaces. */
ra_status rollout_attn_extend(ra_ctx *ctx, const ra_extend *extend, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ROLLOUT_ATTN_CHUNK_H */
