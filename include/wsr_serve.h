/*
 * wsr_serve.h - what serving requests adds to a batched decode step, on AMD Instinct MI355X (gfx950): the C ABI of
 * libwsr_serve.so.
 *
 * Requests come, grow by a token or a few drafts at a time, and go; their keys and values lie in pages of a pool.
 * Beside the operators of wsr_step.h stand
 *   wsr_append_qkv        the projections' fp32 outputs into queries, keys and values: norms of each head, rotary
 *                         positions, 16 bits, keys and values appended to the paged cache
 *   wsr_paged_attention   attention of each sequence's newest tokens over its pages
 *   wsr_token_logprobs    log probabilities of given tokens, with rank, entropy and the most likely alternatives
 *
 * The conventions are wsr_step.h's: every call returns a wsr_status and only enqueues work on `stream`; arguments are
 * checked before anything is enqueued; nothing is allocated, freed or retained; workspaces need no initialisation and may
 * not be shared by calls that overlap; results are deterministic; no call aborts.  Strides are in bytes, >= 0.  Arrays
 * described as `device` hold values the host does not see, so a captured graph may be replayed with other lengths, pages
 * or tokens; values out of their range are clamped or ignored as described and never lead to an access outside the
 * described arrays.
 */
#ifndef WSR_SERVE_H
#define WSR_SERVE_H

#include "wsr_step.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Message describing the last failed call of this header's functions on this thread ("" if none). */
const char* wsr_serve_last_error(void);

/* ---- a paged cache -------------------------------------------------------------------------------

   Key head h of slot s of page p lies at k (v) + p * page_stride + s * tok_stride + h * head_stride, head_dim 16-bit
   values one after another.  Place i of sequence b is slot i % page_size of page table[b][i / page_size]
   (device int32, rows table_stride apart).  A page index outside [0, n_pages) is a hole: nothing is stored there, and its
   keys take part in no attention.  Sequences may share pages that none of them appends to.
   page_size: 1 to 2^20, any number; max_pages (entries of a row): max_pages * page_size <= 2^31 - 4096;
   n_pages < 2^31; k, v 16-byte aligned (null where n_pages is 0), strides multiples of 16, of 4 for the table's. */
typedef struct wsr_pages {
    void *k, *v;
    int64_t page_stride, tok_stride, head_stride;
    int32_t n_pages, page_size;
    const int32_t* table;
    int64_t table_stride;
    int32_t max_pages;
    int32_t reserved;             /* 0 */
} wsr_pages;

/* ---- queries, keys and values of new tokens ------------------------------------------------------

   Sequence b's new tokens are rows starts[b] .. starts[b + 1] - 1 of q, k and v (starts null: one each, row b); they are
   the last n_b of its lens[b] places, so that token i goes to place lens[b] - n_b + i.  For each token and head:
     u = norm(x)     WSR_QKV_NORM: queries and keys, over the head's values, kinds, weights and biases as in wsr_block
                     (weights of queries and of keys, [head_dim]; null: 1 and 0); else u = x
     pair j < rot_dim / 2, (a, b) = u at (j, j + rot_dim / 2), or WSR_QKV_PAIRS at (2 j, 2 j + 1), queries and keys:
                     (a cos t - b sin t, b cos t + a sin t),  t = positions[axis_of[j]][token] * freqs[j]
   Values from rot_dim on pass, and the value heads whole.  Queries are stored to q_out, keys and values to their place
   in the cache, each rounded once to `fmt`; arithmetic is fp32, angles are exact and reduced to a part of a turn right to 2^-50
   while they come to less than 2^45, so that a position of 2^31 turns as exactly as one of 1.
   positions: device int32 (n_axes, n_tokens), or null: the token's place (n_axes 1).  axis_of: device int32
   [rot_dim / 2], clamped to [0, n_axes), or null (all 0).  freqs: device fp32 [rot_dim / 2].
   Tokens of no sequence, and places below 0, past the table's row or in holes, are not stored, and nothing else is
   changed; a token's query does not depend on its place being there.  Two tokens in the same slot, the one case whose result is
   not the same every time, leave some values of each there.  A norm's squares past fp32's range are infinite, its head 0.
   q may be null (nothing but the cache), or k and v (nothing but queries; the cache may be all 0).
   head_dim 64, 128 or 256; rot_dim % 8 == 0, at most head_dim; n_axes 1 to 4; n_tokens and n_seqs at most 2^20, n_heads
   at most 4096 (n_kv_heads too; neither need divide the other here); inputs, weights and q_out 16-byte aligned,
   their strides multiples of 16 (4 for pos_axis_stride).  Outputs overlap nothing. */
#define WSR_QKV_NORM 1
#define WSR_QKV_PAIRS 2
typedef struct wsr_qkv {
    int32_t fmt, flags, kind;
    float eps;
    int32_t n_heads, n_kv_heads, head_dim, rot_dim, n_axes, n_seqs, n_tokens;
    int32_t reserved;             /* 0 */
    const float* q;               /* (n_tokens, n_heads, head_dim), heads one after another */
    int64_t q_tok_stride;
    const float* k;
    int64_t k_tok_stride;
    const float* v;
    int64_t v_tok_stride;
    const void *q_w, *q_b, *k_w, *k_b;
    const float* freqs;
    const int32_t *axis_of, *positions;
    int64_t pos_axis_stride;
    const int32_t *starts, *lens; /* device int32 [n_seqs + 1], not decreasing, clamped to [0, n_tokens]; [n_seqs], from 0 */
    void* q_out;
    int64_t q_out_tok_stride, q_out_head_stride;
    wsr_pages cache;
} wsr_qkv;
wsr_status wsr_append_qkv(const wsr_qkv* p, void* stream);

/* ---- attention of new tokens over a paged cache --------------------------------------------------

   Sequence b's query tokens are rows starts[b] .. starts[b + 1] - 1 of q (starts null: one each, row b), the last n_b of
   its lens[b] places: query i sees keys j < lens[b] - n_b + i + 1 on pages that are no holes,
     out = sum_k softmax_k(scale q . key_k) value_k,  lse = log sum_k exp(scale q . key_k).
   A row that sees no key, or none with a score above -inf, gets out = 0 and lse = -inf, one with a NaN (or +inf) among its
   scores NaN in both; keys past lens[b] and in holes are never read into a result.  Query head h reads key head
   h / (n_heads / n_kv_heads).  Types `fmt`; scores, softmax statistics and sums are fp32, probabilities are rounded to `fmt`
   for the product with the values, out once to `fmt`.
   Rows of q that belong to no sequence (before starts[0], from starts[n_seqs] on) keep what out and lse held.
   starts: device int32 [n_seqs + 1], not decreasing, clamped to [0, n_tokens]; lens: device int32 [n_seqs], clamped to
   [0, max_len]; max_len <= max_pages * page_size.  n_tokens and n_seqs at most 2^20, n_heads at most 4096, tokens
   times heads at most 2^25; n_kv_heads * (n_seqs + a key head's rows / 16) past 2^23 may be refused.  head_dim 64, 128
   or 256; every pointer 16-byte aligned and every stride a multiple of 16 (of 4 for table, starts, lens and lse); lse
   (n_tokens, n_heads) or null; out and lse overlap nothing.  Sums of probabilities, relative to within 2^8 of the largest,
   times values are infinite past fp32's range.  scale is above 0 and at most 2^127.
   Tiles of rows are as high as the call's mean sequence fills: many sequences without tokens beside a few long chunks cost
   time, and are better left out.
   ws: wsr_paged_workspace_bytes(), 256-byte aligned; what it gives serves calls of fewer tokens too where the rest is the
   same (without starts, of fewer sequences). */
typedef struct wsr_paged {
    int32_t fmt, n_heads, n_kv_heads, head_dim, n_seqs, n_tokens;
    float scale;
    int32_t reserved;             /* 0 */
    int64_t max_len;
    const void* q;
    int64_t q_tok_stride, q_head_stride;
    const int32_t *starts, *lens;
    void* out;
    int64_t out_tok_stride, out_head_stride;
    float* lse;
    wsr_pages cache;
} wsr_paged;
size_t wsr_paged_workspace_bytes(const wsr_paged* p);
wsr_status wsr_paged_attention(const wsr_paged* p, void* ws, size_t ws_bytes, void* stream);

/* ---- log probabilities ----------------------------------------------------------------------------

   Of each row of logits, with p = softmax(logits / T), T = temperature[r] (null: 1; T = 0, infinite logits and NaN as in
   wsr_verify: a NaN counts as -inf, +inf as sharing all of the probability, T = 0 and what is not above 0 puts all of it on
   the lowest index of the largest logit, T above 1e30 is 1e30, below 2^-126 is 2^-126):
     logp[r]      log p of tokens[r]                      rank[r]     how many tokens come before it
     entropy[r]   - sum p log p
     top[r]       the n_top tokens that come first, in order, and top_logp[r] their log p
   All of it in fp32: differences of logits past its range are infinite.
   Tokens come in the order of their logits, the larger first, equal ones (-0 and 0 too) by their index.  A token that
   cannot be drawn (logit -inf or NaN) has logp -inf and the rank its place in that order gives; one outside [0, vocab) has
   logp -inf and rank -1.  A row with fewer than n_top tokens that can be drawn ends with token -1 and logp -inf; a row
   with none has entropy 0.
   logits: fp32, 4-byte aligned, row_stride a multiple of 4; tokens: device int32 [n_rows] or null (no logp, no rank);
   logp, rank, entropy and top_logp may be null.  1 <= vocab <= 2^24, 0 <= n_top <= 64, n_rows <= 2^20,
   n_rows * vocab <= 2^40.
   ws: wsr_logprobs_workspace_bytes(), 256-byte aligned; what it gives serves calls of fewer rows too. */
typedef struct wsr_logprobs {
    int64_t n_rows, vocab;
    int32_t n_top;
    int32_t reserved;             /* 0 */
    const float* logits;
    int64_t row_stride;
    const int32_t* tokens;
    const float* temperature;
    float* logp;
    int32_t* rank;
    float* entropy;
    int32_t* top;                 /* (n_rows, n_top) */
    float* top_logp;
} wsr_logprobs;
size_t wsr_logprobs_workspace_bytes(const wsr_logprobs* p);
wsr_status wsr_token_logprobs(const wsr_logprobs* p, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* WSR_SERVE_H */
