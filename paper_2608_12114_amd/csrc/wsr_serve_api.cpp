/*
 * wsr_serve_api.cpp - the C ABI of libwsr_serve (declared in include/wsr_serve.h): argument checks and error
 * reporting.  Every check runs before anything is enqueued and makes no HIP call.
 */
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "wsr_serve_internal.h"

namespace {

thread_local char g_err[512] = "";

wsr_status fail(wsr_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return st;
}

wsr_status done(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(WSR_E_HIP, "%s: launch: %s", what, hipGetErrorString(e));
    g_err[0] = '\0';
    return WSR_OK;
}

bool aligned(const void* p, uintptr_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

/* a * b fits int64 (both >= 0), three such products and a base too. */
bool mul_fits(int64_t a, int64_t b) { return (__int128)a * b <= INT64_MAX / 8; }

struct Stride {
    int64_t bytes, count;       /* count: how many steps of it are addressed */
    const char* name;
};

/* Every stride >= 0, a multiple of `unit` and addressable. */
wsr_status check_strides(std::initializer_list<Stride> all, int64_t unit, const char* who) {
    for (const Stride& s : all) {
        if (s.bytes < 0 || s.bytes % unit)
            return fail(WSR_E_ALIGN, "%s: %s=%lld must be >= 0 and a multiple of %lld", who, s.name, (long long)s.bytes, (long long)unit);
        if (!mul_fits(s.bytes, s.count)) return fail(WSR_E_SIZE, "%s: %s overflows", who, s.name);
    }
    return WSR_OK;
}

wsr_status check_align(std::initializer_list<const void*> all, uintptr_t unit, const char* who) {
    for (const void* p : all)
        if (!aligned(p, unit)) return fail(WSR_E_ALIGN, "%s: %p must be %zu-byte aligned", who, p, (size_t)unit);
    return WSR_OK;
}

bool half_fmt(int32_t f) { return f == WSR_F16 || f == WSR_BF16; }
bool head_dim_fits(int32_t d) { return d == 64 || d == 128 || d == 256; }

#define WSR_TRY(x)                         \
    do {                                   \
        const wsr_status st_ = (x);        \
        if (st_ != WSR_OK) return st_;     \
    } while (0)

wsr_status check_workspace(const void* ws, size_t bytes, size_t need, const char* who) {
    if (!ws) return fail(WSR_E_ARG, "%s: null workspace", who);
    if (!aligned(ws, 256)) return fail(WSR_E_ALIGN, "%s: workspace must be 256-byte aligned", who);
    if (bytes < need) return fail(WSR_E_SIZE, "%s: workspace %zu < %zu bytes", who, bytes, need);
    return WSR_OK;
}

/* The most places of a table's row, and keys of a sequence: counted in 32 bits, rounded up to whole blocks. */
constexpr int64_t MOST_PLACES = INT32_MAX - 4095;

/* The sizes and strides of a cache that sequences of n_seqs read or are appended to. */
wsr_status check_pages(const wsr_pages& c, int64_t n_seqs, int64_t n_kv_heads, const char* who) {
    if (c.n_pages < 0 || c.max_pages < 0 || c.reserved) return fail(WSR_E_ARG, "%s: cache: negative size", who);
    if (c.page_size < 1 || c.page_size > 1 << 20) return fail(WSR_E_SIZE, "%s: page_size=%d must be 1 to 2^20", who, c.page_size);
    if ((int64_t)c.max_pages * c.page_size > MOST_PLACES) return fail(WSR_E_SIZE, "%s: more than 2^31 - 4096 places of a sequence", who);
    WSR_TRY(check_strides({{c.page_stride, c.n_pages, "page_stride"}, {c.tok_stride, c.page_size, "tok_stride"},
                           {c.head_stride, n_kv_heads, "head_stride"}}, 16, who));
    WSR_TRY(check_strides({{c.table_stride, n_seqs, "table_stride"}}, 4, who));
    WSR_TRY(check_align({c.k, c.v}, 16, who));
    WSR_TRY(check_align({c.table}, 4, who));
    if ((c.n_pages > 0 && (!c.k || !c.v)) || (c.max_pages > 0 && n_seqs > 0 && !c.table))
        return fail(WSR_E_ARG, "%s: cache: null pointer", who);
    return WSR_OK;
}

}  // namespace

extern "C" {

const char* wsr_serve_last_error(void) { return g_err; }

/* ---------------------------------- queries, keys and values ----------------------------------- */

wsr_status wsr_append_qkv(const wsr_qkv* p, void* stream) {
    const char* who = "append_qkv";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    if (!half_fmt(p->fmt)) return fail(WSR_E_ARG, "%s: format must be WSR_F16 or WSR_BF16", who);
    if (p->flags & ~(WSR_QKV_NORM | WSR_QKV_PAIRS) || p->reserved) return fail(WSR_E_ARG, "%s: unknown flags %#x", who, p->flags);
    if (p->kind != WSR_NORM_RMS && p->kind != WSR_NORM_LAYER) return fail(WSR_E_ARG, "%s: unknown kind %d", who, p->kind);
    if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return fail(WSR_E_ARG, "%s: eps must be >= 0", who);
    if (!head_dim_fits(p->head_dim)) return fail(WSR_E_SIZE, "%s: head_dim=%d must be 64, 128 or 256", who, p->head_dim);
    if (p->rot_dim < 0 || p->rot_dim % 8 || p->rot_dim > p->head_dim)
        return fail(WSR_E_SIZE, "%s: rot_dim=%d must be a multiple of 8, at most head_dim", who, p->rot_dim);
    if (p->n_axes < 1 || p->n_axes > 4) return fail(WSR_E_ARG, "%s: n_axes=%d must be 1 to 4", who, p->n_axes);
    if (p->n_heads < 0 || p->n_kv_heads < 0 || p->n_seqs < 0 || p->n_tokens < 0) return fail(WSR_E_ARG, "%s: negative size", who);
    if (p->n_heads > 4096 || p->n_kv_heads > 4096 || p->n_seqs > 1 << 20 || p->n_tokens > 1 << 20)
        return fail(WSR_E_SIZE, "%s: too many heads, tokens or sequences", who);
    if (!p->k != !p->v) return fail(WSR_E_ARG, "%s: k and v go together", who);
    if (!p->starts && p->n_tokens != p->n_seqs) return fail(WSR_E_ARG, "%s: without starts each sequence has one token", who);
    const int64_t n = p->n_tokens, D = p->head_dim;
    WSR_TRY(check_strides({{p->q_tok_stride, n, "q_tok_stride"}, {p->k_tok_stride, n, "k_tok_stride"},
                           {p->v_tok_stride, n, "v_tok_stride"}, {p->q_out_tok_stride, n, "q_out_tok_stride"},
                           {p->q_out_head_stride, p->n_heads, "q_out_head_stride"}}, 16, who));
    WSR_TRY(check_strides({{p->pos_axis_stride, p->n_axes, "pos_axis_stride"}}, 4, who));
    WSR_TRY(check_align({p->q, p->k, p->v, p->q_w, p->q_b, p->k_w, p->k_b, p->q_out}, 16, who));
    WSR_TRY(check_align({p->freqs, p->axis_of, p->positions, p->starts, p->lens}, 4, who));
    const wsr_pages& c = p->cache;
    const bool cached = p->k && p->n_kv_heads > 0;
    if (cached || c.table) WSR_TRY(check_pages(c, p->n_seqs, p->n_kv_heads, who));
    if (n == 0 || ((!p->q || !p->n_heads) && !cached)) return done(hipSuccess, who);
    if (p->q && p->n_heads && !p->q_out) return fail(WSR_E_ARG, "%s: null q_out", who);
    if (p->rot_dim && !p->freqs) return fail(WSR_E_ARG, "%s: null freqs", who);
    if (p->n_axes > 1 && p->rot_dim && !p->positions) return fail(WSR_E_ARG, "%s: several axes need positions", who);
    if (!p->lens || p->n_seqs == 0) return fail(WSR_E_ARG, "%s: tokens of no sequence, or null lens", who);
    if (p->q && p->n_heads && ((p->n_heads > 1 && p->q_out_head_stride < 2 * D) || (n > 1 && p->q_out_tok_stride < 2 * D)))
        return fail(WSR_E_ARG, "%s: rows of q_out overlap", who);
    if (cached && ((p->n_kv_heads > 1 && c.head_stride < 2 * D) || (c.page_size > 1 && c.tok_stride < 2 * D) ||
                   (c.n_pages > 1 && c.page_stride < 2 * D)))
        return fail(WSR_E_ARG, "%s: rows of the cache overlap", who);
    return done(wsr_serve::launch_append(*p, static_cast<hipStream_t>(stream)), who);
}

/* ---------------------------------- attention -------------------------------------------------- */

static wsr_status check_paged(const wsr_paged& p, const char* who) {
    if (!half_fmt(p.fmt)) return fail(WSR_E_ARG, "%s: format must be WSR_F16 or WSR_BF16", who);
    if (!head_dim_fits(p.head_dim)) return fail(WSR_E_SIZE, "%s: head_dim=%d must be 64, 128 or 256", who, p.head_dim);
    if (p.n_kv_heads < 1 || p.n_heads < p.n_kv_heads || p.n_heads % p.n_kv_heads || p.n_heads > 4096)
        return fail(WSR_E_ARG, "%s: n_heads=%d must be a multiple of n_kv_heads=%d, at most 4096", who, p.n_heads, p.n_kv_heads);
    if (p.n_seqs < 0 || p.n_tokens < 0 || p.max_len < 0 || p.reserved) return fail(WSR_E_ARG, "%s: negative size", who);
    if (p.n_tokens > 1 << 20 || p.n_seqs > 1 << 20) return fail(WSR_E_SIZE, "%s: too many tokens or sequences", who);
    if ((int64_t)p.n_tokens * p.n_heads > 1 << 25) return fail(WSR_E_SIZE, "%s: tokens times heads above 2^25", who);
    /* the kernels take powers of two: scale log2 e is finite too */
    if (!(p.scale > 0.f) || !std::isfinite(p.scale * 1.4426950408889634f))
        return fail(WSR_E_ARG, "%s: scale must be positive, and finite times log2 e", who);
    if (!p.starts && p.n_tokens != p.n_seqs) return fail(WSR_E_ARG, "%s: without starts each sequence has one token", who);
    if (p.n_seqs == 0 && p.n_tokens > 0) return fail(WSR_E_ARG, "%s: tokens of no sequence", who);
    WSR_TRY(check_pages(p.cache, p.n_seqs, p.n_kv_heads, who));
    if (p.max_len > (int64_t)p.cache.max_pages * p.cache.page_size)
        return fail(WSR_E_SIZE, "%s: max_len=%lld is more than max_pages hold", who, (long long)p.max_len);
    if (!wsr_serve::paged_fits(p)) return fail(WSR_E_SIZE, "%s: too many sequences and key heads for one launch", who);
    return WSR_OK;
}

size_t wsr_paged_workspace_bytes(const wsr_paged* p) {
    if (!p || check_paged(*p, "paged_workspace") != WSR_OK) return 0;
    return wsr_serve::paged_workspace(*p);
}

wsr_status wsr_paged_attention(const wsr_paged* p, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "paged_attention";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_paged(*p, who));
    WSR_TRY(check_strides({{p->q_tok_stride, p->n_tokens, "q_tok_stride"}, {p->q_head_stride, p->n_heads, "q_head_stride"},
                           {p->out_tok_stride, p->n_tokens, "out_tok_stride"}, {p->out_head_stride, p->n_heads, "out_head_stride"}},
                          16, who));
    WSR_TRY(check_align({p->q, p->out}, 16, who));
    WSR_TRY(check_align({p->starts, p->lens, p->lse}, 4, who));
    if (p->n_tokens == 0) return done(hipSuccess, who);
    if (!p->q || !p->out || !p->lens) return fail(WSR_E_ARG, "%s: null pointer", who);
    const int64_t row = 2 * p->head_dim;
    if ((p->n_heads > 1 && p->out_head_stride < row) || (p->n_tokens > 1 && p->out_tok_stride < row))
        return fail(WSR_E_ARG, "%s: rows of out overlap", who);
    WSR_TRY(check_workspace(ws, ws_bytes, wsr_serve::paged_workspace(*p), who));
    return done(wsr_serve::launch_paged(*p, ws, static_cast<hipStream_t>(stream)), who);
}

/* ---------------------------------- log probabilities ------------------------------------------ */

static wsr_status check_logprobs(const wsr_logprobs& p, const char* who) {
    if (p.n_rows < 0 || p.vocab < 1 || p.n_top < 0 || p.reserved) return fail(WSR_E_ARG, "%s: negative size or empty vocabulary", who);
    if (p.n_top > 64) return fail(WSR_E_SIZE, "%s: n_top=%d is above 64", who, p.n_top);
    if (p.vocab > 1 << 24 || p.n_rows > 1 << 20 || p.n_rows * p.vocab > (int64_t)1 << 40)
        return fail(WSR_E_SIZE, "%s: vocab or n_rows too large", who);
    return WSR_OK;
}

size_t wsr_logprobs_workspace_bytes(const wsr_logprobs* p) {
    if (!p || check_logprobs(*p, "logprobs_workspace") != WSR_OK) return 0;
    return wsr_serve::logprobs_workspace(*p);
}

wsr_status wsr_token_logprobs(const wsr_logprobs* p, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "token_logprobs";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_logprobs(*p, who));
    WSR_TRY(check_strides({{p->row_stride, p->n_rows, "row_stride"}}, 4, who));
    WSR_TRY(check_align({p->logits, p->tokens, p->temperature, p->logp, p->rank, p->entropy, p->top, p->top_logp}, 4, who));
    if (p->n_rows == 0) return done(hipSuccess, who);
    if (!p->logits || (p->n_top && !p->top)) return fail(WSR_E_ARG, "%s: null pointer", who);
    if (!p->tokens && (p->logp || p->rank)) return fail(WSR_E_ARG, "%s: logp or rank without tokens", who);
    WSR_TRY(check_workspace(ws, ws_bytes, wsr_serve::logprobs_workspace(*p), who));
    return done(wsr_serve::launch_logprobs(*p, ws, static_cast<hipStream_t>(stream)), who);
}

}  // extern "C"
