/*
 * wsr_step_api.cpp - the C ABI of libwsr_step (declared in include/wsr_step.h): argument checks and error
 * reporting.  Every check runs before anything is enqueued and makes no HIP call.
 */
#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>

#include "wsr_step_internal.h"

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

/* a * b fits int64 (both >= 0). */
bool mul_fits(int64_t a, int64_t b) { return (__int128)a * b <= INT64_MAX / 2; }

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

}  // namespace

extern "C" {

const char* wsr_step_last_error(void) { return g_err; }

/* ---------------------------------- block norm ------------------------------------------------ */

wsr_status wsr_block_norm(const wsr_block* p, void* stream) {
    const char* who = "block_norm";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    if (p->kind != WSR_NORM_RMS && p->kind != WSR_NORM_LAYER) return fail(WSR_E_ARG, "%s: unknown kind %d", who, p->kind);
    if (!half_fmt(p->fmt)) return fail(WSR_E_ARG, "%s: format must be WSR_F16 or WSR_BF16", who);
    if (p->flags & ~WSR_BLOCK_POST || p->reserved) return fail(WSR_E_ARG, "%s: unknown flags %#x", who, p->flags);
    if (p->n_tokens < 0 || p->d < 0) return fail(WSR_E_ARG, "%s: negative size", who);
    if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return fail(WSR_E_ARG, "%s: eps must be >= 0", who);
    if (p->d % 8) return fail(WSR_E_ALIGN, "%s: d=%lld must be a multiple of 8", who, (long long)p->d);
    if (p->d > 32768) return fail(WSR_E_SIZE, "%s: d=%lld is above 32768", who, (long long)p->d);
    if (p->n_tokens > INT32_MAX) return fail(WSR_E_SIZE, "%s: too many tokens", who);
    WSR_TRY(check_strides({{p->y_tok_stride, p->n_tokens, "y_tok_stride"}, {p->gate_tok_stride, p->n_tokens, "gate_tok_stride"},
                           {p->h_tok_stride, p->n_tokens, "h_tok_stride"}, {p->h_out_tok_stride, p->n_tokens, "h_out_tok_stride"},
                           {p->x_tok_stride, p->n_tokens, "x_tok_stride"}}, 16, who));
    WSR_TRY(check_align({p->y, p->post_w, p->post_b, p->gate, p->h, p->h_out, p->pre_w, p->pre_b, p->x}, 16, who));
    if (p->n_tokens == 0 || p->d == 0) return done(hipSuccess, who);
    if (!p->y && !p->h) return fail(WSR_E_ARG, "%s: neither y nor h", who);
    if (!p->h_out && !p->x) return fail(WSR_E_ARG, "%s: neither h_out nor x", who);
    if (p->n_tokens > 1) {
        if (p->h_out && p->h_out_tok_stride < 4 * p->d) return fail(WSR_E_ARG, "%s: rows of h_out overlap", who);
        if (p->x && p->x_tok_stride < 2 * p->d) return fail(WSR_E_ARG, "%s: rows of x overlap", who);
        if (p->h_out && p->h_out == p->h && p->h_tok_stride != p->h_out_tok_stride)
            return fail(WSR_E_ARG, "%s: h_out in place of h needs the same stride", who);
    }
    return done(wsr_step::launch_block_norm(*p, static_cast<hipStream_t>(stream)), who);
}

/* ---------------------------------- adapters -------------------------------------------------- */

static wsr_status check_loras(const wsr_lora* mods, int32_t n, int32_t n_tokens, const char* who) {
    if (n < 0 || n_tokens < 0) return fail(WSR_E_ARG, "%s: n=%d n_tokens=%d", who, n, n_tokens);
    if (n_tokens > 1 << 20) return fail(WSR_E_SIZE, "%s: more than 2^20 tokens", who);
    if (n > 0 && !mods) return fail(WSR_E_ARG, "%s: null pointer", who);
    for (int32_t i = 0; i < n; ++i) {
        const wsr_lora& m = mods[i];
        char at[64];
        std::snprintf(at, sizeof at, "%s: projection %d", who, i);
        if (!half_fmt(m.fmt)) return fail(WSR_E_ARG, "%s: format must be WSR_F16 or WSR_BF16", at);
        if (m.rank < 1 || m.rank > 256) return fail(WSR_E_ARG, "%s: rank=%d must be 1 to 256", at, m.rank);
        if (m.M < 0 || m.K < 0) return fail(WSR_E_ARG, "%s: negative size M=%lld K=%lld", at, (long long)m.M, (long long)m.K);
        if (m.M > INT32_MAX || m.K > (1 << 28)) return fail(WSR_E_SIZE, "%s: M or K too large", at);
        if (m.K % 8) return fail(WSR_E_ALIGN, "%s: K=%lld must be a multiple of 8", at, (long long)m.K);
        WSR_TRY(check_strides({{m.a_stride, 8192, "a_stride"}, {m.x_tok_stride, n_tokens, "x_tok_stride"}}, 16, at));
        WSR_TRY(check_strides({{m.b_stride, 8192, "b_stride"}}, 2, at));
        WSR_TRY(check_strides({{m.y0_tok_stride, n_tokens, "y0_tok_stride"}, {m.y_tok_stride, n_tokens, "y_tok_stride"}}, 4, at));
        WSR_TRY(check_align({m.a, m.x}, 16, at));
        WSR_TRY(check_align({m.b}, 2, at));
        WSR_TRY(check_align({m.y, m.y0}, 4, at));
        if (m.M == 0 || n_tokens == 0) continue;
        if (!m.y || (m.K > 0 && (!m.a || !m.x)) || !m.b) return fail(WSR_E_ARG, "%s: null pointer", at);
        if (n_tokens > 1 && m.y_tok_stride < 4 * m.M) return fail(WSR_E_ARG, "%s: tokens would share outputs (y_tok_stride < 4 M)", at);
        if (m.y0 == m.y && n_tokens > 1 && m.y0_tok_stride != m.y_tok_stride)
            return fail(WSR_E_ARG, "%s: y0 in place of y needs the same stride", at);
    }
    int64_t rows = 0;
    for (int32_t i = 0; i < n; ++i) rows += mods[i].M;
    if (rows > (int64_t)1 << 36) return fail(WSR_E_SIZE, "%s: more than 2^36 rows", who);
    return WSR_OK;
}

size_t wsr_lora_workspace_bytes(const wsr_lora* mods, int32_t n, int32_t n_tokens) {
    if (!mods || n <= 0 || n_tokens <= 0 || n_tokens > 1 << 20) return 0;
    for (int32_t i = 0; i < n; ++i)
        if (mods[i].rank < 1 || mods[i].rank > 256 || mods[i].K < 0 || mods[i].K > (1 << 28)) return 0;
    return wsr_step::lora_workspace(mods, n, n_tokens);
}

wsr_status wsr_lora_sweep(const wsr_lora* mods, int32_t n, int32_t n_tokens, const int32_t* adapter_of, int32_t n_adapters,
                          const int32_t* ranks, const float* scales, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "lora_sweep";
    WSR_TRY(check_loras(mods, n, n_tokens, who));
    if (n_adapters < 0 || n_adapters > 8192) return fail(WSR_E_SIZE, "%s: n_adapters=%d must be 0 to 8192", who, n_adapters);
    WSR_TRY(check_align({adapter_of, ranks, scales}, 4, who));
    if (n == 0 || n_tokens == 0) return done(hipSuccess, who);
    if (!adapter_of) return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_workspace(ws, ws_bytes, wsr_step::lora_workspace(mods, n, n_tokens), who));
    return done(wsr_step::launch_lora(mods, n, n_tokens, adapter_of, n_adapters, ranks, scales, ws, static_cast<hipStream_t>(stream)), who);
}

/* ---------------------------------- attention ------------------------------------------------- */

static wsr_status check_attn(const wsr_attn& p, const char* who) {
    if (!half_fmt(p.fmt)) return fail(WSR_E_ARG, "%s: format must be WSR_F16 or WSR_BF16", who);
    if (p.head_dim != 64 && p.head_dim != 128) return fail(WSR_E_SIZE, "%s: head_dim=%d must be 64 or 128", who, p.head_dim);
    if (p.n_kv_heads < 1 || p.n_heads < p.n_kv_heads || p.n_heads % p.n_kv_heads || p.n_heads > 4096)
        return fail(WSR_E_ARG, "%s: n_heads=%d must be a multiple of n_kv_heads=%d, at most 4096", who, p.n_heads, p.n_kv_heads);
    if (p.n_seqs < 0 || p.n_tokens < 0 || p.prefix_len < 0 || p.max_len < 0 || p.reserved)
        return fail(WSR_E_ARG, "%s: negative size", who);
    if (p.n_tokens > 1 << 20 || p.n_seqs > 1 << 20 || p.prefix_len > 1 << 30 || p.max_len > 1 << 30)
        return fail(WSR_E_SIZE, "%s: too many tokens, sequences or keys", who);
    /* the whole form counts a row's keys, rounded up to whole parts and blocks, in 32 bits */
    if (p.prefix_len + p.max_len > INT32_MAX - 4095) return fail(WSR_E_SIZE, "%s: more than 2^31 - 4096 keys of a row", who);
    if ((int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads) > 1 << 30) return fail(WSR_E_SIZE, "%s: more than 2^30 rows of a key head", who);
    if (!(p.scale > 0.f) || !std::isfinite(p.scale)) return fail(WSR_E_ARG, "%s: scale must be positive and finite", who);
    if (!p.starts && p.n_tokens != p.n_seqs) return fail(WSR_E_ARG, "%s: without starts each sequence has one token", who);
    if (p.n_seqs == 0 && p.n_tokens > 0) return fail(WSR_E_ARG, "%s: tokens of no sequence", who);
    if (!wsr_step::attn_fits(p)) return fail(WSR_E_SIZE, "%s: too many sequences and key heads for one launch", who);
    return WSR_OK;
}

size_t wsr_attn_workspace_bytes(const wsr_attn* p) {
    if (!p || check_attn(*p, "attn_workspace") != WSR_OK) return 0;
    return wsr_step::attn_workspace(*p);
}

wsr_status wsr_prefix_attention(const wsr_attn* p, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "prefix_attention";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_attn(*p, who));
    WSR_TRY(check_strides({{p->q_tok_stride, p->n_tokens, "q_tok_stride"}, {p->q_head_stride, p->n_heads, "q_head_stride"},
                           {p->prefix_tok_stride, p->prefix_len, "prefix_tok_stride"},
                           {p->prefix_head_stride, p->n_kv_heads, "prefix_head_stride"},
                           {p->kv_seq_stride, p->n_seqs, "kv_seq_stride"}, {p->kv_tok_stride, p->max_len, "kv_tok_stride"},
                           {p->kv_head_stride, p->n_kv_heads, "kv_head_stride"},
                           {p->out_tok_stride, p->n_tokens, "out_tok_stride"}, {p->out_head_stride, p->n_heads, "out_head_stride"}},
                          16, who));
    if (p->prefix_tok_stride > 16 << 20 || p->kv_tok_stride > 16 << 20)
        return fail(WSR_E_SIZE, "%s: strides between keys above 16 MiB", who);
    WSR_TRY(check_align({p->q, p->k_prefix, p->v_prefix, p->k, p->v, p->out}, 16, who));
    WSR_TRY(check_align({p->starts, p->lens, p->lse}, 4, who));
    if (p->n_tokens == 0) return done(hipSuccess, who);
    if (!p->q || !p->out || !p->lens || (p->prefix_len && (!p->k_prefix || !p->v_prefix)) || (p->max_len && (!p->k || !p->v)))
        return fail(WSR_E_ARG, "%s: null pointer", who);
    const int64_t row = 2 * p->head_dim;
    if ((p->n_heads > 1 && p->out_head_stride < row) || (p->n_tokens > 1 && p->out_tok_stride < row))
        return fail(WSR_E_ARG, "%s: rows of out overlap", who);
    WSR_TRY(check_workspace(ws, ws_bytes, wsr_step::attn_workspace(*p), who));
    return done(wsr_step::launch_attn(*p, ws, static_cast<hipStream_t>(stream)), who);
}

/* ---------------------------------- verification ---------------------------------------------- */

static wsr_status check_verify(const wsr_verify& p, const char* who) {
    if (p.n_seqs < 0 || p.n_drafts < 0 || p.vocab < 1) return fail(WSR_E_ARG, "%s: negative size or empty vocabulary", who);
    if (p.n_drafts > 63) return fail(WSR_E_SIZE, "%s: n_drafts=%d is above 63", who, p.n_drafts);
    if (p.vocab > 1 << 24 || p.n_seqs > 1 << 16) return fail(WSR_E_SIZE, "%s: vocab or n_seqs too large", who);
    return WSR_OK;
}

size_t wsr_verify_workspace_bytes(const wsr_verify* p) {
    if (!p || check_verify(*p, "verify_workspace") != WSR_OK) return 0;
    return wsr_step::verify_workspace(*p);
}

wsr_status wsr_verify_drafts(const wsr_verify* p, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "verify_drafts";
    if (!p) return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_verify(*p, who));
    WSR_TRY(check_strides({{p->target_seq_stride, p->n_seqs, "target_seq_stride"},
                           {p->target_row_stride, p->n_drafts + 1, "target_row_stride"},
                           {p->draft_seq_stride, p->n_seqs, "draft_seq_stride"}, {p->draft_row_stride, p->n_drafts, "draft_row_stride"},
                           {p->noise_seq_stride, p->n_seqs, "noise_seq_stride"}}, 4, who));
    WSR_TRY(check_align({p->target, p->draft, p->tokens, p->counts, p->temperature, p->uniform, p->noise, p->out, p->accepted,
                         p->logp}, 4, who));
    if (p->n_seqs == 0) return done(hipSuccess, who);
    if (!p->target || !p->noise || !p->out || !p->accepted || (p->n_drafts && (!p->tokens || !p->uniform)))
        return fail(WSR_E_ARG, "%s: null pointer", who);
    WSR_TRY(check_workspace(ws, ws_bytes, wsr_step::verify_workspace(*p), who));
    return done(wsr_step::launch_verify(*p, ws, static_cast<hipStream_t>(stream)), who);
}

}  // extern "C"
