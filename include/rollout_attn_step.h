/*
 * rollout_attn, both ends of a step: the places of its new tokens before the
 * layers, the verification of its drafts and the next tokens after them.
 *
 * Setting.  A step of a rollout worker (rollout_attn.h, rollout_attn_chunk.h)
 * takes, for every sequence, some new tokens: one, a turn, a draft of a few
 * that are checked at once.  Before the layers each new token needs a page and
 * a slot; after them the drafted tokens are held against the target's
 * probabilities, and every sequence gets its next token:
 *   rollout_attn_place     takes pages from a stack of free ones where the
 *                          sequences need them, and writes the block table, the
 *                          packed offsets, positions and slots of the new tokens;
 *   rollout_attn_verify    accepts drafted tokens in order (speculative sampling)
 *                          and draws one token a sequence; without drafts it is
 *                          the choice of the next token;
 *   rollout_attn_release   puts pages that sequences no longer need back.
 * Lengths, tables and counts stay on the device, so that a whole step can be
 * recorded into one HIP graph.  Responses end at lengths of high variance (paper
 * Sec. 7.4), so pages come and go all the time; the paper leaves this to its
 * inference engine (Sec. 2.1.1); this header defines it.
 *
 * Contexts, streams, ownership of memory, status codes and error texts are
 * those of rollout_attn.h: no call allocates, copies or waits, each enqueues
 * kernels on the given stream and nothing else, and so may be recorded into a HIP
 * graph; inputs may be reused or freed once the stream has passed the call.
 * Results are deterministic: the same inputs give the same bytes.
 */
#ifndef ROLLOUT_ATTN_STEP_H
#define ROLLOUT_ATTN_STEP_H

#include "rollout_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Places of new tokens.  Sequence b holds L = seq_lens[b] tokens in the first held[b] pages of its block-table row and asks for
 * n = new_tokens[b] more.  F is the number of pages of its prompt group's prefix (the optional hint of ra_problem; 0 without
 * one), H = max(held[b], F), P = ceil((L + n) / page_size) pages are needed, and M = max(0, P - H) of them come from the stack
 * free_pages[0 .. *free_count), the last one first, for sequences in their order and for a sequence's pages in theirs.
 *   Not considered: n <= 0; L or held[b] negative; held[b], F or P beyond max_pages_per_seq; L > page_size * H.
 *   Served is a considered sequence if
 *     M == 0, or the M of all considered sequences up to b, itself included, add up to at most *free_count, and
 *     the n of all considered sequences up to b add up to at most total_tokens.
 *   (So the first sequence for whose pages the stack is too low, and those behind it that need pages, get nothing; those that
 *   have room in their pages go on.)
 * A served sequence:
 *   block_table[b][i]   prefix_pages[prefix_page_offsets[g] + i] for held[b] <= i < F, pages from the stack for H <= i < P;
 *                       all others are left as they are
 *   held_out[b]         max(H, P)            lens_out[b]  L + n
 * Any other: its row is left as it is, held_out[b] = held[b], lens_out[b] = seq_lens[b], and it has no tokens.  For all:
 *   cu_seqlens          int32 [num_seqs + 1], first token of each sequence among the new ones, packed; [num_seqs] is their total
 *   *free_count_out     *free_count less the pages taken (the stack's entries stay as they are)
 *   positions[t]        of the t-th new token: its place in its sequence, L + i            (NULL: not written)
 *   slots[t]            page * page_size + place in the page, the row of a pool laid out [page][slot] (NULL: not written)
 *   seqs[t]             its sequence                                                          (NULL: not written)
 *   -1 in positions, slots and seqs for total <= t < total_tokens: rollout_attn_rotate and rollout_attn_append_chunk leave out
 *   tokens of such positions, so a captured step may have room for more tokens than it has.
 * seq_lens and lens_out, held and held_out, free_count and free_count_out may be the same memory; otherwise outputs overlap
 * nothing.  *free_count counts as the nearest of 0 and num_pages outside them.  Page ids are not looked into.
 * Supported: page_size == 16; num_seqs * max_pages_per_seq < 2^31; num_seqs < 2^31 - 1024; max_pages_per_seq < 2^27.
 */
typedef struct {
    int32_t num_seqs, total_tokens, page_size, num_pages, max_pages_per_seq;
    const int32_t *seq_lens;     /* dev [num_seqs] */
    const int32_t *new_tokens;   /* dev [num_seqs] */
    const int32_t *held;         /* dev [num_seqs] */
    const int32_t *free_pages;   /* dev [num_pages] */
    const int32_t *free_count;   /* dev [1] */
    int32_t num_groups;
    const int32_t *seq_group;           /* dev [num_seqs] or NULL when num_groups == 0; -1: no group */
    const int32_t *prefix_page_offsets; /* dev [num_groups + 1] or NULL when num_groups == 0 */
    const int32_t *prefix_pages;        /* dev or NULL when num_groups == 0 */
    int32_t *block_table;        /* dev [num_seqs][max_pages_per_seq] */
    int32_t *cu_seqlens;         /* dev [num_seqs + 1] */
    int32_t *lens_out;           /* dev [num_seqs] */
    int32_t *held_out;           /* dev [num_seqs] */
    int32_t *free_count_out;     /* dev [1] */
    int32_t *positions;          /* dev [total_tokens] or NULL */
    int64_t *slots;              /* dev [total_tokens] or NULL */
    int32_t *seqs;               /* dev [total_tokens] or NULL */
} ra_place;

/* Host-only check of the scalars and pointers (device data is not read): what rollout_attn_place would return for them
 * before touching the device.  msg (may be NULL) receives a NUL-terminated explanation. */
ra_status rollout_attn_check_place(const ra_place *place, char *msg, size_t msg_len);

/* Enqueues the placing: one kernel; two where many tokens may come and lengths or counts are written where they are read. */
ra_status rollout_attn_place(ra_ctx *ctx, const ra_place *place, void *hip_stream);

/*
 * Pages back to the stack.  Sequence b keeps its first keep_lens[b] tokens (less than 0 counts as 0) and the K = min(held[b],
 * ceil(keep_lens[b] / page_size)) pages that they are in: held_out[b] = K, and the pages block_table[b][max(K, F) .. held[b])
 * go onto the stack, for sequences in their order and for a sequence's pages in theirs, F being the pages of its group's
 * prefix: those belong to the group, and whoever took them for it gives them back.  *free_count_out is *free_count and what
 * was put on; entries that would lie past num_pages are not written, nor counted.  Sequences whose held[b] is negative or beyond
 * max_pages_per_seq keep what they have.  block_table is not changed.  held and held_out, free_count and free_count_out may
 * be the same memory.  A page must not come back twice; nothing checks this.
 * Supported: as for ra_place.
 */
typedef struct {
    int32_t num_seqs, page_size, num_pages, max_pages_per_seq;
    const int32_t *keep_lens;    /* dev [num_seqs] */
    const int32_t *held;         /* dev [num_seqs] */
    const int32_t *block_table;  /* dev [num_seqs][max_pages_per_seq] */
    int32_t num_groups;
    const int32_t *seq_group;           /* dev [num_seqs] or NULL when num_groups == 0; -1: no group */
    const int32_t *prefix_page_offsets; /* dev [num_groups + 1] or NULL when num_groups == 0 */
    int32_t *free_pages;         /* dev [num_pages] */
    const int32_t *free_count;   /* dev [1] */
    int32_t *held_out;           /* dev [num_seqs] */
    int32_t *free_count_out;     /* dev [1] */
} ra_release;

ra_status rollout_attn_check_release(const ra_release *release, char *msg, size_t msg_len);

/* Enqueues the release: one kernel; two where many pages may come back and counts are written where they are read. */
ra_status rollout_attn_release(ra_ctx *ctx, const ra_release *release, void *hip_stream);

typedef enum { RA_LOGITS_BF16 = 0, RA_LOGITS_FP32 = 1 } ra_logits_dtype;

/*
 * Verification of drafted tokens, and the next token of every sequence.  Sequence b has the rows t = cu_rows[b] ..
 * cu_rows[b+1] - 1 of logits: row t is the target's at a token that the step took in, and tokens[t + 1] for t + 1 < cu_rows[b+1]
 * is the drafted token that row t judges (so tokens and cu_rows are what the step was called with: the last token of the
 * sequence and its drafts; tokens[cu_rows[b]] does not count).  The last row judges none.  With T = temperature[b],
 *   p_t = softmax(logits[t] / T),   q_t = softmax(draft_logits[draft_rows[b] + t - cu_rows[b]] / T)
 * where q_t is the distribution that tokens[t + 1] was drawn from; without draft_logits it is all on that token (a guess from
 * the text so far, a greedy draft).  In order, the draft x = tokens[t + 1] of row t is accepted if
 *   accept_uniform[t] * q_t(x) < p_t(x),
 * until one is not; accepted[b] is the number that were.  Then one token is drawn, by the number draw_uniform[b] = v, from the
 * weights w of the row t that comes next, cu_rows[b] + accepted[b]:
 *   w = p_t                    if t is the last row,
 *   w = max(p_t - q_t, 0)      if its draft was turned down (without draft_logits: p_t without x); p_t if that is all zeros,
 * the token being the first one i with w_0 + .. + w_i > v * (w_0 + .. + w_{V-1}).  (With numbers that are independent and even on
 * [0, 1) every token is then distributed as if sampled from p alone.)  All of this is as in binary64, so that the sums of many small
 * weights move no border: with weights that are right to 2^-38; or, in large batches, with sums of binary32 weights where what they
 * may be off by settles the comparison, and in binary64 for the tests and draws that they leave open.
 *   T == 0 (or less, or NaN): greedy.  p_t is all on the largest logit, the first of equals; draft_logits are not read: a draft is
 *   accepted if it is that token.  T counts as the nearest of 1e-30 and 1e30 outside them.
 *   out_tokens[t]     for the sequence's rows: the accepted drafts, then the token drawn, then -1
 *   out_logprobs[t]   ln p_t(out_tokens[t]), 0 where out_tokens[t] is -1; rounded to binary32, and off by 2^-17 at most where sums
 *                     were of binary32 weights.  Whether they were goes by the size of the batch: the same row's may differ by
 *                     that much from one batch to another                                  (NULL: not written)
 *   next_tokens[b]    the token drawn                                                      (NULL: not written)
 * Logits of -inf have probability 0, whatever masks them; a row that has a NaN or +inf in it, or nothing but -inf, has no
 * distribution: p_t of such a row accepts no draft, and the token drawn from it is -1, with a log-probability of NaN; q_t of such a
 * row, a draft row outside [0, total_draft_rows) or a draft that is no token (not in [0, vocab)) has the draft turned down and
 * the token drawn from p_t.  v outside [0, 1] counts as the nearest of the two, NaN as 0.
 * A sequence without rows (one that asked for no tokens, or that rollout_attn_place did not serve): accepted[b] = 0,
 * next_tokens[b] = -1.  Rows behind cu_rows[num_seqs] are left as they were in the outputs.  cu_rows starts at 0 or more and does not
 * decrease; a sequence whose rows are not in [0, total_rows] counts as having none.
 * Of what the step put into the cache, accepted[b] + 1 tokens stay, the one that it began with and the accepted drafts; but none of a
 * sequence without rows: whoever keeps lengths adds that where cu_rows[b+1] > cu_rows[b] alone.
 * Layout: element (t, i) of logits at t * logits_stride + i, V = vocab values in a row, aligned to an element; draft_logits alike.
 * 16-byte aligned rows are read fastest.  Inputs and outputs overlap nothing.
 * A probability below 2^-990 counts as 0.
 * Supported: vocab <= 2^24; num_seqs and total_rows <= 2^22; with a row's parts of 4096 values, total_rows (twice that with
 * draft_logits) times those fewer than 2^26, and num_seqs times those fewer than 2^32.
 */
typedef struct {
    int32_t num_seqs, total_rows, vocab;
    int32_t logits_dtype;          /* ra_logits_dtype */
    const void *logits;            /* dev */
    int64_t logits_stride;         /* in elements, at least vocab */
    const int32_t *cu_rows;        /* dev [num_seqs + 1] */
    const int32_t *tokens;         /* dev [total_rows]; needed, as accept_uniform is, also where no sequence has a draft */
    const void *draft_logits;      /* dev or NULL */
    int64_t draft_stride;
    int32_t draft_dtype;           /* ra_logits_dtype */
    int32_t total_draft_rows;
    const int32_t *draft_rows;     /* dev [num_seqs], or NULL without draft_logits: a sequence's first row of them */
    const float *temperature;      /* dev [num_seqs], or NULL: 1 */
    const float *accept_uniform;   /* dev [total_rows]; a sequence's last does not count, the array's last is not read */
    const float *draw_uniform;     /* dev [num_seqs] */
    int32_t *accepted;             /* dev [num_seqs] */
    int32_t *out_tokens;           /* dev [total_rows] */
    float *out_logprobs;           /* dev [total_rows] or NULL */
    int32_t *next_tokens;          /* dev [num_seqs] or NULL */
} ra_verify;

ra_status rollout_attn_check_verify(const ra_verify *verify, char *msg, size_t msg_len);

/* Bytes of device workspace rollout_attn_verify needs for this shape (only num_seqs, total_rows, vocab, logits_dtype, and whether
 * draft_logits is NULL are read).  ctx may be NULL: the size for a 256-compute-unit device is returned. */
ra_status rollout_attn_verify_workspace_size(const ra_ctx *ctx, const ra_verify *shape_only, size_t *bytes);

/* Enqueues the verification on hip_stream: two kernels, one more with draft_logits and one more in large batches.  The environment's
 * ROLLOUT_ATTN_VERIFY_FEW=n, read by rollout_attn_create, is the number of bf16 logits up to which all sums are binary64 from the
 * start, of binary32 logits five times as many, and n / 680 more for every sequence; with a draft model's logits (both counted) n / 2 and
 * 5 n / 4.  The default is 2^24.  workspace as for rollout_attn_decode: dev memory of at least
 * rollout_attn_verify_workspace_size() bytes, 256-byte aligned, contents irrelevant on entry and undefined afterwards; calls
 * that overlap in time need distinct workspaces. */
ra_status rollout_attn_verify(ra_ctx *ctx, const ra_verify *verify, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* ROLLOUT_ATTN_STEP_H */
