// C-ABI of the operators for chunks of new tokens (see include/rollout_attn_chunk.h): argument checks, launches.
#include "../../include/rollout_attn_chunk.h"
#include "ra_chunk.h"
#include "ra_context.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

using ra::set_err;

namespace {

// A failed check: its status, and its text in msg.
struct Fail {
    char *msg;
    size_t n;
    __attribute__((format(printf, 3, 4))) ra_status operator()(ra_status st, const char *fmt, ...) const
    {
        if (msg && n) {
            va_list ap;
            va_start(ap, fmt);
            vsnprintf(msg, n, fmt, ap);
            va_end(ap);
        }
        return st;
    }
};

ra_status check_rows(const ra_rotate *p, const Fail &fail, bool append)
{
    if (p->num_tokens < 0 || p->Hq < 0 || p->Hkv < 0 || p->D <= 0 || p->Hq > 65536 || p->Hkv > 65536)
        return fail(RA_ERR_INVALID_ARG, "dimension out of range (num_tokens=%d Hq=%d Hkv=%d D=%d)", p->num_tokens, p->Hq, p->Hkv, p->D);
    if (p->D != 64 && p->D != 128) return fail(RA_ERR_UNSUPPORTED, "D=%d (only 64 and 128 are supported)", p->D);
    if (p->rot_dim < 0 || p->rot_dim > p->D) return fail(RA_ERR_INVALID_ARG, "rot_dim=%d is not in 0 .. D", p->rot_dim);
    if ((p->q_weight || p->k_weight) && !(std::isfinite(p->eps) && p->eps >= 0.f))
        return fail(RA_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (p->rot_dim % 16) return fail(RA_ERR_UNSUPPORTED, "rot_dim=%d (only multiples of 16 are supported)", p->rot_dim);
    if (p->num_tokens == 0) return RA_OK;
    auto tensor = [&](const char *name, const void *x, int64_t stride, int heads) -> ra_status {
        if (!x) return fail(RA_ERR_INVALID_ARG, "a required pointer (%s) is NULL", name);
        if ((uintptr_t)x % 16) return fail(RA_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
        if (stride % 8 || stride < (int64_t)heads * p->D)
            return fail(RA_ERR_INVALID_ARG, "the stride of %s must be a multiple of 8 elements and at least heads * D", name);
        if (stride > (int64_t)1 << 40) return fail(RA_ERR_UNSUPPORTED, "the stride of %s is too large", name);
        return RA_OK;
    };
    ra_status st = RA_OK;
    if (p->q && p->Hq > 0) {
        st = tensor("q", p->q, p->q_stride_token, p->Hq);
        if (st == RA_OK) st = tensor("q_out", p->q_out, p->q_out_stride_token, p->Hq);
    }
    if (st == RA_OK && (append || p->k) && p->Hkv > 0) {
        st = tensor("k", p->k, p->k_stride_token, p->Hkv);
        if (st == RA_OK && !append) st = tensor("k_out", p->k_out, p->k_out_stride_token, p->Hkv);
    }
    if (st != RA_OK) return st;
    if (append && p->k_out) return fail(RA_ERR_INVALID_ARG, "an append writes keys to the cache: k_out must be NULL");
    if (((uintptr_t)p->q_weight | (uintptr_t)p->k_weight) % 16) return fail(RA_ERR_INVALID_ARG, "q_weight and k_weight must be 16-byte aligned");
    if (p->rot_dim > 0) {
        if (!p->rope || (!append && !p->positions)) return fail(RA_ERR_INVALID_ARG, "a rotation needs rope%s", append ? "" : " and positions");
        if (p->rope_len < 0) return fail(RA_ERR_INVALID_ARG, "rope_len is negative");
        if ((uintptr_t)p->rope % 16) return fail(RA_ERR_INVALID_ARG, "rope must be 16-byte aligned");
    }
    return RA_OK;
}

// The cache of an append or of the attention of chunks.
template <typename P> ra_status check_cache(const P *p, int Hkv, int D, int64_t tokens, const Fail &fail)
{
    if (p->num_seqs < 0 || p->max_chunk_len < 0 || p->page_size <= 0 || p->num_pages < 0 || p->max_pages_per_seq < 0)
        return fail(RA_ERR_INVALID_ARG, "negative or zero dimension (num_seqs=%d max_chunk_len=%d page_size=%d num_pages=%d max_pages_per_seq=%d)",
                    p->num_seqs, p->max_chunk_len, p->page_size, p->num_pages, p->max_pages_per_seq);
    if (p->kv_dtype != RA_KV_BF16 && p->kv_dtype != RA_KV_FP8_E4M3) return fail(RA_ERR_INVALID_ARG, "kv_dtype=%d is not a ra_kv_dtype", p->kv_dtype);
    if (p->page_size != 16) return fail(RA_ERR_UNSUPPORTED, "page_size=%d (only 16 is supported)", p->page_size);
    if ((int64_t)p->num_seqs * p->max_pages_per_seq >= (int64_t)1 << 31 || p->max_pages_per_seq > INT32_MAX / 16 ||
        (tokens + 2 * (int64_t)p->num_seqs) * (2 * (int64_t)Hkv) >= (int64_t)1 << 31)
        return fail(RA_ERR_UNSUPPORTED, "batch too large");
    if (p->num_seqs == 0 || tokens == 0) return RA_OK;
    if (!p->cu_seqlens || !p->seq_lens || !p->block_table || !p->k_pool || !p->v_pool)
        return fail(RA_ERR_INVALID_ARG, "a required pointer (cu_seqlens, seq_lens, block_table, k_pool, v_pool) is NULL");
    const int es = p->kv_dtype == RA_KV_FP8_E4M3 ? 1 : 2;
    if (p->kv_stride_token < D || p->kv_stride_head < 0 || p->kv_stride_page < 0)
        return fail(RA_ERR_INVALID_ARG, "kv strides must be non-negative and kv_stride_token >= D");
    if ((p->kv_stride_token * es) % 16 || (p->kv_stride_head * es) % 16 || (p->kv_stride_page * es) % 16)
        return fail(RA_ERR_INVALID_ARG, "kv strides must be multiples of 16 bytes");
    if (p->kv_stride_token > INT32_MAX / 32) return fail(RA_ERR_UNSUPPORTED, "kv_stride_token too large");
    if (((uintptr_t)p->k_pool | (uintptr_t)p->v_pool) % 16) return fail(RA_ERR_INVALID_ARG, "k_pool and v_pool must be 16-byte aligned");
    if (es == 1 && (!p->k_scale || !p->v_scale)) return fail(RA_ERR_INVALID_ARG, "fp8 KV needs k_scale and v_scale");
    return RA_OK;
}

ra_status check_rotate(const ra_rotate *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "rotate is NULL");
    return check_rows(p, fail, false);
}

ra_status check_append(const ra_append_chunk *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "append is NULL");
    if (p->rot.Hkv <= 0) return fail(RA_ERR_INVALID_ARG, "negative or zero dimension (Hkv=%d)", p->rot.Hkv);
    ra_status st = check_rows(&p->rot, fail, true);
    if (st == RA_OK) st = check_cache(p, p->rot.Hkv, p->rot.D, p->rot.num_tokens, fail);
    if (st != RA_OK || p->num_seqs == 0 || p->rot.num_tokens == 0) return st;
    if (!p->v) return fail(RA_ERR_INVALID_ARG, "a required pointer (v) is NULL");
    if ((uintptr_t)p->v % 16) return fail(RA_ERR_INVALID_ARG, "v must be 16-byte aligned");
    if (p->v_stride_token % 8 || p->v_stride_token < (int64_t)p->rot.Hkv * p->rot.D)
        return fail(RA_ERR_INVALID_ARG, "the stride of v must be a multiple of 8 elements and at least heads * D");
    if (p->v_stride_token > (int64_t)1 << 40) return fail(RA_ERR_UNSUPPORTED, "the stride of v is too large");
    return RA_OK;
}

ra_status check_extend(const ra_extend *p, char *msg, size_t n)
{
    const Fail fail = {msg, n};
    if (msg && n) msg[0] = 0;
    if (!p) return fail(RA_ERR_INVALID_ARG, "extend is NULL");
    if (p->total_tokens < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->D <= 0)
        return fail(RA_ERR_INVALID_ARG, "negative or zero dimension (total_tokens=%d Hq=%d Hkv=%d D=%d)", p->total_tokens, p->Hq, p->Hkv, p->D);
    if (p->Hq % p->Hkv) return fail(RA_ERR_INVALID_ARG, "Hq=%d is not a multiple of Hkv=%d", p->Hq, p->Hkv);
    if (!std::isfinite(p->softmax_scale) || p->softmax_scale <= 0.f) return fail(RA_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
    if (p->D != 64 && p->D != 128) return fail(RA_ERR_UNSUPPORTED, "D=%d (only 64 and 128 are supported)", p->D);
    if (p->Hq / p->Hkv > 128) return fail(RA_ERR_UNSUPPORTED, "Hq/Hkv=%d (at most 128 is supported)", p->Hq / p->Hkv);
    ra_status st = check_cache(p, p->Hkv, p->D, p->total_tokens, fail);
    if (st != RA_OK) return st;
    // 32-bit row numbers inside a sequence, and a stream of work (32 keys of a block of rows to a unit) below 2^30 units
    const int64_t rows = (int64_t)p->max_chunk_len * (p->Hq / p->Hkv);
    const int64_t blocks = (int64_t)p->total_tokens * (p->Hq / p->Hkv) / 128 + p->num_seqs;
    if (rows >= (int64_t)1 << 30 || blocks * p->Hkv >= (int64_t)1 << 23 || blocks * p->Hkv * ((int64_t)p->max_pages_per_seq / 2 + 16) >= (int64_t)1 << 30)
        return fail(RA_ERR_UNSUPPORTED, "batch too large");
    if (p->num_seqs == 0 || p->total_tokens == 0 || p->max_chunk_len == 0) return RA_OK;
    if (!p->q || !p->out || !p->lse) return fail(RA_ERR_INVALID_ARG, "a required pointer (q, out, lse) is NULL");
    if (((uintptr_t)p->q | (uintptr_t)p->out) % 16 || (uintptr_t)p->lse % 4)
        return fail(RA_ERR_INVALID_ARG, "q and out must be 16-byte aligned, lse 4-byte aligned");
    if (p->q_stride_token % 8 || p->q_stride_token < (int64_t)p->Hq * p->D)
        return fail(RA_ERR_INVALID_ARG, "the stride of q must be a multiple of 8 elements and at least heads * D");
    if (p->q_stride_token > (int64_t)1 << 40) return fail(RA_ERR_UNSUPPORTED, "the stride of q is too large");
    return RA_OK;
}

void fill_rows(ra::RowsLaunch &a, const ra_rotate *p)
{
    memset(&a, 0, sizeof a);
    a.T = p->num_tokens, a.D = p->D;
    a.Hq = p->q ? p->Hq : 0, a.Hkv = p->k ? p->Hkv : 0;
    a.q = (const uint16_t *)p->q, a.k = (const uint16_t *)p->k;
    a.q_out = (uint16_t *)p->q_out, a.k_out = (uint16_t *)p->k_out;
    a.q_stride = p->q_stride_token, a.k_stride = p->k_stride_token;
    a.q_out_stride = p->q_out_stride_token, a.k_out_stride = p->k_out_stride_token;
    a.qw = p->q_weight, a.kw = p->k_weight, a.eps = p->eps;
    a.rope_len = p->rope_len, a.rot = p->rot_dim, a.interleaved = p->interleaved != 0;
    if (a.rot) a.positions = p->positions, a.rope = p->rope;
}

void fill_shape(ra::ExtendLaunch &a, const ra_extend *p, int num_cus)
{
    a.B = p->num_seqs, a.T = p->total_tokens, a.max_chunk = p->max_chunk_len;
    a.Hq = p->Hq, a.Hkv = p->Hkv, a.D = p->D, a.G = p->Hq / p->Hkv;
    a.max_pages = p->max_pages_per_seq, a.num_cus = num_cus;
}

// One new token for every sequence, in a shape that the decode step has: what it is asked then, if q is contiguous.
bool as_decode(const ra_extend *p, ra_problem &d)
{
    if (p->max_chunk_len != 1 || p->total_tokens != p->num_seqs || p->Hq / p->Hkv > 16) return false;
    memset(&d, 0, sizeof d);
    d.B = p->num_seqs, d.Hq = p->Hq, d.Hkv = p->Hkv, d.D = p->D, d.page_size = p->page_size, d.num_pages = p->num_pages;
    d.max_pages_per_seq = p->max_pages_per_seq;
    d.q = p->q, d.k_pool = p->k_pool, d.v_pool = p->v_pool;
    d.kv_stride_page = p->kv_stride_page, d.kv_stride_head = p->kv_stride_head, d.kv_stride_token = p->kv_stride_token;
    d.kv_dtype = p->kv_dtype, d.k_scale = p->k_scale, d.v_scale = p->v_scale;
    d.block_table = p->block_table, d.seq_lens = p->seq_lens;
    d.softmax_scale = p->softmax_scale, d.out = p->out, d.lse = p->lse;
    return true;
}

// Runs `launch` on the context's device.
template <typename F> ra_status on_device(ra_ctx *c, F launch)
{
    int prev = 0;
    hipError_t e = hipGetDevice(&prev);
    if (e == hipSuccess && prev != c->device) e = hipSetDevice(c->device);
    if (e == hipSuccess) e = launch();
    if (prev != c->device) (void)hipSetDevice(prev);
    if (e != hipSuccess) { set_err(c, "HIP: %s", hipGetErrorString(e)); return RA_ERR_DEVICE; }
    return RA_OK;
}

} // namespace

extern "C" {

ra_status rollout_attn_check_rotate(const ra_rotate *p, char *msg, size_t n) { return check_rotate(p, msg, n); }
ra_status rollout_attn_check_append_chunk(const ra_append_chunk *p, char *msg, size_t n) { return check_append(p, msg, n); }
ra_status rollout_attn_check_extend(const ra_extend *p, char *msg, size_t n) { return check_extend(p, msg, n); }

ra_status rollout_attn_rotate(ra_ctx *c, const ra_rotate *p, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_rotate(p, c->err, sizeof c->err);
    if (st != RA_OK || p->num_tokens == 0) return st;
    ra::RowsLaunch a;
    fill_rows(a, p);
    return on_device(c, [&] { return ra::launch_rotate(a, c->num_cus, (hipStream_t)stream); });
}

ra_status rollout_attn_append_chunk(ra_ctx *c, const ra_append_chunk *p, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_append(p, c->err, sizeof c->err);
    if (st != RA_OK || p->num_seqs == 0 || p->rot.num_tokens == 0 || p->max_chunk_len == 0) return st;
    ra::RowsLaunch a;
    fill_rows(a, &p->rot);
    const int es = p->kv_dtype == RA_KV_FP8_E4M3 ? 1 : 2;
    a.v = (const uint16_t *)p->v, a.v_stride = p->v_stride_token;
    a.B = p->num_seqs, a.max_chunk = p->max_chunk_len, a.max_pages = p->max_pages_per_seq, a.num_pages = p->num_pages;
    a.cu = p->cu_seqlens, a.seq_lens = p->seq_lens, a.table = p->block_table;
    a.k_pool = (uint8_t *)p->k_pool, a.v_pool = (uint8_t *)p->v_pool;
    a.stride_page_b = p->kv_stride_page * es, a.stride_head_b = p->kv_stride_head * es, a.stride_token_b = (int32_t)(p->kv_stride_token * es);
    a.k_scale = p->k_scale, a.v_scale = p->v_scale;
    return on_device(c, [&] { return ra::launch_append_chunk(a, es == 1, c->num_cus, (hipStream_t)stream); });
}

ra_status rollout_attn_extend_workspace_size(const ra_ctx *c, const ra_extend *p, size_t *bytes)
{
    ra_ctx *const err = const_cast<ra_ctx *>(c);
    if (!p || !bytes) { set_err(err, "extend or bytes is NULL"); return RA_ERR_INVALID_ARG; }
    if (p->num_seqs < 0 || p->total_tokens < 0 || p->max_chunk_len < 0 || p->max_pages_per_seq < 0 || p->Hq <= 0 || p->Hkv <= 0 || p->Hq % p->Hkv) {
        set_err(err, "bad shape for a workspace query");
        return RA_ERR_INVALID_ARG;
    }
    if ((p->D != 64 && p->D != 128) || p->Hq / p->Hkv > 128) {
        set_err(err, "unsupported shape for a workspace query (D in {64,128}, Hq/Hkv <= 128)");
        return RA_ERR_UNSUPPORTED;
    }
    ra::ExtendLaunch a;
    memset(&a, 0, sizeof a);
    fill_shape(a, p, c ? c->num_cus : 256);
    *bytes = ra::carve_extend(a, nullptr);
    ra_problem d;
    size_t n = 0;
    if (as_decode(p, d) && rollout_attn_workspace_size(c, &d, &n) == RA_OK && n > *bytes) *bytes = n;
    return RA_OK;
}

ra_status rollout_attn_extend(ra_ctx *c, const ra_extend *p, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!c) { set_err(nullptr, "ctx is NULL"); return RA_ERR_INVALID_ARG; }
    const ra_status st = check_extend(p, c->err, sizeof c->err);
    if (st != RA_OK || p->num_seqs == 0 || p->total_tokens == 0 || p->max_chunk_len == 0) return st;
    size_t need = 0;
    const ra_status sized = rollout_attn_extend_workspace_size(c, p, &need);
    if (sized != RA_OK) return sized;
    if (need && (!workspace || ((uintptr_t)workspace & 255))) { set_err(c, "workspace is NULL or not 256-byte aligned"); return RA_ERR_INVALID_ARG; }
    if (workspace_bytes < need) {
        set_err(c, "workspace of %zu bytes given, %zu needed", workspace_bytes, need);
        return RA_ERR_WORKSPACE_TOO_SMALL;
    }
    ra_problem d;
    if (p->q_stride_token == (int64_t)p->Hq * p->D && as_decode(p, d) && rollout_attn_check_problem(&d, nullptr, 0) == RA_OK)
        return rollout_attn_decode(c, &d, workspace, workspace_bytes, stream);
    const int es = p->kv_dtype == RA_KV_FP8_E4M3 ? 1 : 2;
    ra::ExtendLaunch a;
    memset(&a, 0, sizeof a);
    fill_shape(a, p, c->num_cus);
    (void)ra::carve_extend(a, workspace);
    a.num_pages = p->num_pages, a.kv_fp8 = es == 1;
    a.magic_g = (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G);
    a.q = (const uint16_t *)p->q, a.q_stride = p->q_stride_token;
    a.cu = p->cu_seqlens, a.seq_lens = p->seq_lens, a.table = p->block_table;
    a.k_pool = (const uint8_t *)p->k_pool, a.v_pool = (const uint8_t *)p->v_pool;
    a.stride_page_b = p->kv_stride_page * es, a.stride_head_b = p->kv_stride_head * es, a.stride_token_b = (int32_t)(p->kv_stride_token * es);
    a.k_scale = p->k_scale, a.v_scale = p->v_scale;
    a.scale_log2 = p->softmax_scale * 1.4426950408889634f;
    a.out = (uint16_t *)p->out, a.lse = p->lse, a.zeros = c->zeros;
    return on_device(c, [&] { return ra::launch_extend(a, (hipStream_t)stream); });
}

} // extern "C"
