// C-ABI of both ends of a step (see include/rollout_attn_step.h): argument checks, launches.
#include "../../include/rollout_attn_step.h"
#include "ra_check.h"
#include "ra_step.h"

#include <cstring>

using ra::Fail;
using ra::on_device;
using ra::set_err;

namespace {

// What a place and a release have in common.
template <typename P> ra_status check_pages(const P *p, const Fail &fail)
{
    if (p->num_seqs < 0 || p->page_size <= 0 || p->num_pages < 0 || p->max_pages_per_seq < 0 || p->num_groups < 0)
        return fail(RA_ERR_INVALID_ARG, "negative or zero dimension (num_seqs=%d page_size=%d num_pages=%d max_pages_per_seq=%d num_groups=%d)", p->num_seqs,
                    p->page_size, p->num_pages, p->max_pages_per_seq, p->num_groups);
    if (p->page_size != 16) return fail(RA_ERR_UNSUPPORTED, "page_size=%d (only 16 is supported)", p->page_size);
    if ((int64_t)p->num_seqs * p->max_pages_per_seq >= (int64_t)1 << 31 || p->max_pages_per_seq > INT32_MAX / 16 || p->num_seqs > ra::kMostPagedSeqs)
        return fail(RA_ERR_UNSUPPORTED, "batch too large");
    if (!p->free_count || !p->free_count_out) return fail(RA_ERR_INVALID_ARG, "a required pointer (free_count, free_count_out) is NULL");
    if (p->num_seqs == 0) return RA_OK;
    if (!p->held || !p->held_out) return fail(RA_ERR_INVALID_ARG, "a required pointer (held, held_out) is NULL");
    if (p->max_pages_per_seq > 0 && !p->block_table) return fail(RA_ERR_INVALID_ARG, "a required pointer (block_table) is NULL");
    if (p->num_pages > 0 && !p->free_pages) return fail(RA_ERR_INVALID_ARG, "a required pointer (free_pages) is NULL");
    if (p->num_groups > 0 && (!p->seq_group || !p->prefix_page_offsets))
        return fail(RA_ERR_INVALID_ARG, "a prompt-group hint needs seq_group and prefix_page_offsets");
    return RA_OK;
}

ra_status check_place(const ra_place *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "place is NULL");
    if (p->total_tokens < 0) return fail(RA_ERR_INVALID_ARG, "total_tokens is negative");
    const ra_status st = check_pages(p, fail);
    if (st != RA_OK) return st;
    if (!p->cu_seqlens) return fail(RA_ERR_INVALID_ARG, "a required pointer (cu_seqlens) is NULL");
    if ((uintptr_t)p->slots % 8) return fail(RA_ERR_INVALID_ARG, "slots must be 8-byte aligned");
    if (p->num_seqs == 0) return RA_OK;
    if (!p->seq_lens || !p->new_tokens || !p->lens_out) return fail(RA_ERR_INVALID_ARG, "a required pointer (seq_lens, new_tokens, lens_out) is NULL");
    if (p->num_groups > 0 && !p->prefix_pages) return fail(RA_ERR_INVALID_ARG, "a prompt-group hint needs prefix_pages");
    return RA_OK;
}

ra_status check_release(const ra_release *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "release is NULL");
    const ra_status st = check_pages(p, fail);
    if (st != RA_OK || p->num_seqs == 0) return st;
    if (!p->keep_lens) return fail(RA_ERR_INVALID_ARG, "a required pointer (keep_lens) is NULL");
    return RA_OK;
}

bool is_logits_dtype(int t) { return t == RA_LOGITS_BF16 || t == RA_LOGITS_FP32; }

ra_status check_shape(const ra_verify *p, const Fail &fail)
{
    if (p->num_seqs < 0 || p->total_rows < 0 || p->vocab <= 0)
        return fail(RA_ERR_INVALID_ARG, "negative or zero dimension (num_seqs=%d total_rows=%d vocab=%d)", p->num_seqs, p->total_rows, p->vocab);
    if (p->vocab > 1 << 24) return fail(RA_ERR_UNSUPPORTED, "vocab=%d (at most 2^24 is supported)", p->vocab);
    if (p->num_seqs > 1 << 22 || p->total_rows > 1 << 22 || !ra::verify_fits(p->num_seqs, p->total_rows, p->vocab, p->draft_logits != nullptr))
        return fail(RA_ERR_UNSUPPORTED, "batch too large");
    return RA_OK;
}

ra_status check_verify(const ra_verify *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "verify is NULL");
    const ra_status st = check_shape(p, fail);
    if (st != RA_OK) return st;
    auto tensor = [&](const char *name, const void *x, int64_t stride, int32_t dtype) -> ra_status {
        if (!is_logits_dtype(dtype)) return fail(RA_ERR_INVALID_ARG, "the dtype of %s (%d) is not a ra_logits_dtype", name, dtype);
        if ((uintptr_t)x % (dtype == RA_LOGITS_FP32 ? 4 : 2)) return fail(RA_ERR_INVALID_ARG, "%s must be aligned to an element", name);
        if (stride < p->vocab) return fail(RA_ERR_INVALID_ARG, "the stride of %s must be at least vocab", name);
        if (stride > (int64_t)1 << 32) return fail(RA_ERR_UNSUPPORTED, "the stride of %s is too large", name);
        return RA_OK;
    };
    ra_status t = tensor("logits", p->logits, p->logits_stride, p->logits_dtype);
    if (t == RA_OK && p->draft_logits) {
        if (p->total_draft_rows < 0) return fail(RA_ERR_INVALID_ARG, "total_draft_rows is negative");
        t = tensor("draft_logits", p->draft_logits, p->draft_stride, p->draft_dtype);
    }
    if (t != RA_OK || p->num_seqs == 0) return t;
    if (!p->cu_rows || !p->accepted) return fail(RA_ERR_INVALID_ARG, "a required pointer (cu_rows, accepted) is NULL");
    if (p->total_rows > 0 && (!p->logits || !p->tokens || !p->accept_uniform || !p->draw_uniform || !p->out_tokens))
        return fail(RA_ERR_INVALID_ARG, "a required pointer (logits, tokens, accept_uniform, draw_uniform, out_tokens) is NULL");
    if (p->draft_logits && !p->draft_rows) return fail(RA_ERR_INVALID_ARG, "draft_logits need draft_rows");
    return RA_OK;
}

void fill_shape(ra::VerifyLaunch &a, const ra_verify *p)
{
    memset(&a, 0, sizeof a);
    a.B = p->num_seqs, a.R = p->total_rows, a.V = p->vocab, a.fp32 = p->logits_dtype == RA_LOGITS_FP32;
}

template <typename P> void fill_pages(ra::PagesLaunch &a, const P *p)
{
    memset(&a, 0, sizeof a);
    a.B = p->num_seqs, a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq, a.num_groups = p->num_groups;
    a.held = p->held, a.group = p->seq_group, a.pfx_off = p->prefix_page_offsets;
    a.free_count = p->free_count, a.stack = const_cast<int32_t *>(p->free_pages), a.table = const_cast<int32_t *>(p->block_table);
    a.held_out = p->held_out, a.free_out = p->free_count_out;
}

} // namespace

extern "C" {

ra_status rollout_attn_check_place(const ra_place *p, char *msg, size_t n) { return check_place(p, msg, n); }
ra_status rollout_attn_check_release(const ra_release *p, char *msg, size_t n) { return check_release(p, msg, n); }
ra_status rollout_attn_check_verify(const ra_verify *p, char *msg, size_t n) { return check_verify(p, msg, n); }

ra_status rollout_attn_place(ra_ctx *c, const ra_place *p, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_place(p, c->err, sizeof c->err);
    if (st != RA_OK) return st;
    ra::PagesLaunch a;
    fill_pages(a, p);
    a.T = p->total_tokens, a.lens = p->seq_lens, a.asked = p->new_tokens, a.pfx_pages = p->prefix_pages;
    a.cu = p->cu_seqlens, a.lens_out = p->lens_out, a.positions = p->positions, a.slots = p->slots, a.seqs = p->seqs;
    return on_device(c, [&] { return ra::launch_place(a, c->num_cus, (hipStream_t)stream); });
}

ra_status rollout_attn_release(ra_ctx *c, const ra_release *p, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_release(p, c->err, sizeof c->err);
    if (st != RA_OK) return st;
    ra::PagesLaunch a;
    fill_pages(a, p);
    a.lens = p->keep_lens;
    return on_device(c, [&] { return ra::launch_release(a, c->num_cus, (hipStream_t)stream); });
}

ra_status rollout_attn_verify_workspace_size(const ra_ctx *c, const ra_verify *p, size_t *bytes)
{
    ra_ctx *const err = const_cast<ra_ctx *>(c);
    if (!p || !bytes) { set_err(err, "verify or bytes is NULL"); return RA_ERR_INVALID_ARG; }
    char msg[512];
    const ra_status st = check_shape(p, Fail{msg, sizeof msg});
    if (st != RA_OK) { set_err(err, "%s", msg); return st; }
    ra::VerifyLaunch a;
    fill_shape(a, p);
    *bytes = ra::carve_verify(a, c ? c->num_cus : 256, c ? c->verify_few : ra::kVerifyFew, p->draft_logits != nullptr, nullptr);
    return RA_OK;
}

ra_status rollout_attn_verify(ra_ctx *c, const ra_verify *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_verify(p, c->err, sizeof c->err);
    if (st != RA_OK || p->num_seqs == 0) return st;
    ra::VerifyLaunch a;
    fill_shape(a, p);
    const size_t need = ra::carve_verify(a, c->num_cus, c->verify_few, p->draft_logits != nullptr, workspace);
    if (need && (!workspace || ((uintptr_t)workspace & 255))) { set_err(c, "workspace is NULL or not 256-byte aligned"); return RA_ERR_INVALID_ARG; }
    if (workspace_bytes < need) {
        set_err(c, "workspace of %zu bytes given, %zu needed", workspace_bytes, need);
        return RA_ERR_WORKSPACE_TOO_SMALL;
    }
    a.logits = p->logits, a.stride = p->logits_stride;
    if (p->draft_logits) {
        a.draft_fp32 = p->draft_dtype == RA_LOGITS_FP32, a.draft = p->draft_logits, a.draft_stride = p->draft_stride;
        a.total_draft_rows = p->total_draft_rows, a.draft_rows = p->draft_rows;
    }
    a.cu = p->cu_rows, a.tokens = p->tokens, a.temperature = p->temperature, a.u = p->accept_uniform, a.v = p->draw_uniform;
    a.accepted = p->accepted, a.out = p->out_tokens, a.next = p->next_tokens, a.logprobs = p->out_logprobs;
    return on_device(c, [&] { return ra::launch_verify(a, (hipStream_t)stream); });
}

} // extern "C"
