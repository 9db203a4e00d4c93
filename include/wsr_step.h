/*
 * wsr_step.h - what a batched decode step does between its weight passes, on AMD Instinct MI355X
 * (gfx950): the C ABI of libwsr_step.so.
 *
 * The weight passes of wsr.h take 16-bit activation columns and leave fp32 outputs.  The four
 * operators here stand between them, for single tokens, for the candidates of a speculative step
 * and for prompts:
 *   wsr_block_norm         a block's fp32 outputs back into the residual stream, with the norms after
 *                          and before a block, and the 16-bit activations of the next pass
 *   wsr_lora_sweep         the low-rank adapters of many requests, added to the projections' outputs
 *   wsr_prefix_attention   attention of a batch whose sequences share a long prefix
 *   wsr_verify_drafts      acceptance of drafted tokens against the target's logits, and the next token
 *
 * The conventions are wsr.h's: every call returns a wsr_status and only enqueues work on `stream`
 * (a hipStream_t, NULL for the null stream); arguments are checked before anything is enqueued;
 * nothing is allocated, freed or retained; workspaces need no initialisation and may not be shared by
 * calls that overlap; results are deterministic; no call aborts.  Strides are in bytes, >= 0.  Arrays
 * described as `device` hold values the host does not see, so a captured graph may be replayed with
 * other lengths, adapters or drafts; values out of their range are clamped or ignored as described
 * and never lead to an access outside the described arrays.
 */
#ifndef WSR_STEP_H
#define WSR_STEP_H

#include "wsr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Message describing the last failed call of this header's functions on this thread ("" if none). */
const char* wsr_step_last_error(void);

/* ---- norms around a block, gate and residual scale ---------------------------------------------

   For each token:  v  = post(y)        (WSR_BLOCK_POST; else v = y; no y: v = 0)
                    h' = res_scale * h + gate * v      (no gate: 1; no h: 0)
                    x  = pre(h')        (no x: not computed)
   post and pre are the same kind: WSR_NORM_RMS   u / sqrt(mean(u^2) + eps) * w + b, or
   WSR_NORM_LAYER (u - mean(u)) / sqrt(mean((u - mean(u))^2) + eps) * w + b, with w = 1 and b = 0
   where their pointers are null.  h' is stored to h_out (if not null) in fp32, x is rounded once to
   `fmt` (WSR_F16 or WSR_BF16), the type of w, b and gate too.  All arithmetic is fp32; an infinity or
   NaN in a token's inputs reaches that token's outputs only.
   d % 8 == 0, d <= 32768, n_tokens < 2^31; rows and vectors 16-byte aligned, token strides multiples of
   16.  gate: one vector for all tokens (stride 0) or one per token.  h_out may be h itself (same
   stride); outputs otherwise overlap nothing. */
#define WSR_NORM_RMS 0
#define WSR_NORM_LAYER 1
#define WSR_BLOCK_POST 1
typedef struct wsr_block {
    int32_t kind, fmt, flags;
    float eps, res_scale;
    int32_t reserved;             /* 0 */
    int64_t n_tokens, d;
    const float* y;               /* (n_tokens, d) the block's outputs */
    int64_t y_tok_stride;
    const void *post_w, *post_b;  /* [d] */
    const void* gate;             /* [d] or (n_tokens, d) */
    int64_t gate_tok_stride;
    const float* h;               /* (n_tokens, d) the residual stream */
    int64_t h_tok_stride;
    float* h_out;
    int64_t h_out_tok_stride;
    const void *pre_w, *pre_b;    /* [d] */
    void* x;                      /* (n_tokens, d) activations of the next weight pass */
    int64_t x_tok_stride;
} wsr_block;
wsr_status wsr_block_norm(const wsr_block* p, void* stream);

/* ---- adapters of many requests beside shared projections -----------------------------------------

   For t < n_tokens and each projection m, with a = adapter_of[t] and r = ranks[a]:
     y_m(t) = y0_m(t) + scales[a] * B_m,a (A_m,a x_m(t)),
   A_m,a the first r rows of (rank, K) at a + a * a_stride, B_m,a the first r columns of (M, rank) at
   b + a * b_stride, both row-major in `fmt` (WSR_F16 or WSR_BF16), x in the same type, y and y0 fp32
   (y0 null: 0; y0 may be y itself with the same stride, the usual case after a sweep).  A token whose
   adapter is outside [0, n_adapters) has none: y = y0.  Products are exact, sums are fp32, and the
   inner vector A x enters the second product with 24 bits (WSR_BF16), or with 22 (WSR_F16: entries down
   to 2^-28 of the token's largest; smaller ones within 2^-50 of it).  Rows of A and columns of B from r
   on are not read.
   A projection with M = 0 does nothing and may have null pointers; with K = 0, a and x may be null.
   adapter_of: device int32 [n_tokens], in any order; ranks: device int32 [n_adapters], clamped to
   [0, rank], or null (all `rank`); scales: device fp32 [n_adapters] or null (all 1).
   K % 8 == 0, 1 <= rank <= 256; a, x 16-byte aligned, a_stride and x_tok_stride multiples of 16; b
   2-byte aligned; y, y0 4-byte aligned, strides multiples of 4, y_tok_stride >= 4 M for more than one
   token.  n_tokens <= 2^20, n_adapters <= 8192, M < 2^31, K <= 2^28, 2^36 rows in all.  ws:
   wsr_lora_workspace_bytes(), 256-byte aligned, read and written by this call only. */
typedef struct wsr_lora {
    int32_t fmt, rank;
    int64_t M, K;
    const void* a;
    int64_t a_stride;             /* bytes between adapters */
    const void* b;
    int64_t b_stride;
    const void* x;
    int64_t x_tok_stride;
    const float* y0;
    int64_t y0_tok_stride;
    float* y;
    int64_t y_tok_stride;
} wsr_lora;
size_t wsr_lora_workspace_bytes(const wsr_lora* mods, int32_t n, int32_t n_tokens);
wsr_status wsr_lora_sweep(const wsr_lora* mods, int32_t n, int32_t n_tokens, const int32_t* adapter_of,
                          int32_t n_adapters, const int32_t* ranks, const float* scales, void* ws, size_t ws_bytes,
                          void* stream);

/* ---- attention of a batch behind a shared prefix -----------------------------------------------------

   Sequence b's query tokens are rows starts[b] .. starts[b + 1] - 1 of q (starts null: one token each,
   row b); they are its last n_b of lens[b] own keys.  Query i of sequence b sees all prefix_len keys
   of the prefix and its own keys j < lens[b] - n_b + i + 1:
     out = sum_k softmax_k(scale q . key_k) value_k,  lse = log sum_k exp(scale q . key_k).
   A row that sees no key gets out = 0 and lse = -inf, one with a NaN among its scores NaN in both.  Query
   head h reads key head h / (n_heads / n_kv_heads).  Types `fmt` (WSR_F16 or WSR_BF16); scores, softmax
   statistics and sums are fp32, probabilities are rounded to `fmt` for the product with the values, out
   once to `fmt`.
   Keys past lens[b] are never read into a result (they may hold anything).  Rows of q that belong to no
   sequence (before starts[0], from starts[n_seqs] on) leave unspecified values in out and lse.
   starts: device int32 [n_seqs + 1], not decreasing, starts[n_seqs] <= n_tokens; lens: device int32
   [n_seqs], clamped to [0, max_len].  prefix_len and max_len at most 2^30, together at most 2^31 - 4096;
   n_tokens and n_seqs at most 2^20, n_heads at most 4096, rows of a key head (tokens times its query
   heads) at most 2^30; calls with n_kv_heads * (n_seqs + those rows / 128) past 2^22 may be refused.
   head_dim 64 or 128; every pointer 16-byte aligned and every stride a multiple of 16 (of 4 for lse);
   tok strides of keys at most 16 MiB; lse (n_tokens, n_heads) or null.  k_prefix and v_prefix (k and v)
   have the same strides.  ws: wsr_attn_workspace_bytes(), 256-byte aligned. */
typedef struct wsr_attn {
    int32_t fmt, n_heads, n_kv_heads, head_dim, n_seqs, n_tokens;
    float scale;
    int32_t reserved;             /* 0 */
    const void* q;
    int64_t q_tok_stride, q_head_stride;
    const void *k_prefix, *v_prefix;
    int64_t prefix_len, prefix_tok_stride, prefix_head_stride;
    const void *k, *v;
    int64_t max_len, kv_seq_stride, kv_tok_stride, kv_head_stride;
    const int32_t *starts, *lens;
    void* out;
    int64_t out_tok_stride, out_head_stride;
    float* lse;
} wsr_attn;
size_t wsr_attn_workspace_bytes(const wsr_attn* p);
wsr_status wsr_prefix_attention(const wsr_attn* p, void* ws, size_t ws_bytes, void* stream);

/* ---- verification of drafted tokens ------------------------------------------------------------------

   Sequence b has counts[b] drafted tokens (null: n_drafts), target logits in rows 0 .. counts[b] (row
   i: the distribution of the token after i accepted drafts) and the draft model's logits in rows
   0 .. counts[b] - 1 (draft null: each draft was looked up, its distribution all on that token).
   With p = softmax(target / T), q = softmax(draft / T), T = temperature[b] (null: 1; T = 0, and what is
   not above 0: all on the lowest index of the largest logit; above 1e30: 1e30), drafts are accepted in
   order while uniform_i * q_i(x_i) < p_i(x_i).
   At the first refusal i, or after the last draft, the next token is the index with the largest
   w_v / noise_v (ties: the lowest), w = max(p_i - q_i, 0), after the last draft w = p (and where all
   of w is 0): with Exp(1) noise, a sample in proportion to w.
     out[b]       accepted drafts, the next token, then -1 up to n_drafts + 1 entries
     accepted[b]  how many drafts were accepted
     logp[b]      log p of each emitted token in its row, 0 after the last (null: not stored)
   A NaN logit counts as -inf (a token that cannot be drawn), +inf as sharing all of the probability; a row
   with no token that can be drawn accepts nothing and gives token -1 with logp -inf, and so does a
   draft outside [0, vocab) count as refused.
   target, draft: fp32, strides multiples of 4, rows 4-byte aligned; tokens: int32 (n_seqs, n_drafts);
   uniform: fp32 (n_seqs, n_drafts) in [0, 1); noise: fp32 (n_seqs, vocab), from 2^-126 to
   2^100; counts, temperature: device [n_seqs], counts clamped to [0, n_drafts].  1 <= vocab <= 2^24,
   0 <= n_drafts <= 63, n_seqs <= 2^16.  ws: wsr_verify_workspace_bytes(), 256-byte aligned. */
typedef struct wsr_verify {
    int32_t n_seqs, n_drafts;
    int64_t vocab;
    const float* target;
    int64_t target_seq_stride, target_row_stride;
    const float* draft;
    int64_t draft_seq_stride, draft_row_stride;
    const int32_t *tokens, *counts;
    const float *temperature, *uniform, *noise;
    int64_t noise_seq_stride;
    int32_t *out, *accepted;
    float* logp;
} wsr_verify;
size_t wsr_verify_workspace_bytes(const wsr_verify* p);
wsr_status wsr_verify_drafts(const wsr_verify* p, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* WSR_STEP_H */
