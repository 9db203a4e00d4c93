/*
 * wsr_attn.hip - attention of a batch whose sequences share a prefix.
 *
 * A query row is one (token, query head); the G = n_heads / n_kv_heads heads of a key head and all
 * tokens of the batch stand side by side as rows of one matrix product per key head, so the prefix is
 * read once for all of them.  Every workgroup walks blocks of keys with a running maximum and sum:
 *
 *   S^T = K Q^T   (v_mfma 32x32x16: 32 keys x 32 rows, each lane one row)
 *   P   = exp2((S - max) scale log2 e), O^T += V^T P^T with P still in the registers of S: the lane
 *         layout of S^T is the operand layout of P^T when V's keys are taken in the same order, and
 *         V's transpose comes out of LDS by transposing reads (ds_read_b64_tr_b16).
 *
 * P is rounded to the values' type: as two terms, which would leave the rounding of the output alone, the second
 * product and its operands cost a third of the long cases (4 prompts of up to 900 behind 8192 357 us with one term, 481
 * with two, error against 64 bits 0.0022 and 0.0017 relative; 24 sequences of 5 behind 32771 158 and 201; f16, 4 tokens
 * behind 1024 10.3 and 10.7, 0.00025 and 0.00021).  The sum of a row's probabilities, the maximum and all sums are fp32.
 *
 * Keys and values go from memory straight into LDS, two buffers, the next block in flight while one is
 * worked on; 16-byte pieces are placed so that reads meet no bank twice.
 *
 *  - split form (few rows): workgroups over parts of the prefix for all rows, and over parts of each
 *    sequence's own keys; each leaves a maximum, a sum and an unnormalised fp32 row, which
 *    k_attn_join adds up.
 *  - whole form (prompts): a workgroup takes 128 rows of one sequence through the prefix and its own
 *    keys and stores the result.  The chip holds 512 such workgroups at a time; the last round of them,
 *    where it would leave places empty, is cut into parts along the keys that fill them (a part leaves what
 *    one of the split form does, and k_attn_join_units adds them up).
 *
 * Many rows are bound by the matrix cores and the exponentials between their products: 4 prompts of up to 900 tokens
 * behind 8192 (354 GFLOP) take 352 to 389 us, 910 to 1005 TFLOP/s, where a product of 8192 x 8192 matrices reaches 1200; 24 sequences
 * of 5 tokens behind 32771 (132 GFLOP) 158 to 170 us, 775 to 830 TFLOP/s (a sequence's 40 rows leave most of a row tile over its own
 * keys empty).  Few rows are bound by latency: 4 tokens behind 1024 take 10.3 us, two launches' chains of loads.
 */
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "wsr_attend.h"

namespace wsr_step {

struct AttnPlan {
    int32_t prefix_tiles, prefix_parts;    /* row tiles and key parts of the prefix (split form) */
    int32_t own_tiles, own_parts;          /* most row tiles over all sequences, most key parts of one */
    int32_t own_block;                     /* keys that a workgroup takes at a time */
    int32_t prefix_part;                   /* keys of a part of the prefix */
    int32_t most_parts;                    /* parts of a unit of the whole form's last round, at most */
    float* part;                           /* [(prefix_parts + own_parts)][n_tokens][n_heads][head_dim + 4], or
                                              whole: [HELD][128][head_dim + 4] */
    bool whole;
};

/* The query tokens of sequence b. */
__device__ __forceinline__ int start_of(const wsr_attn& p, int b) {
    return p.starts ? min(max(p.starts[b], 0), p.n_tokens) : min(b, p.n_tokens);
}
__device__ __forceinline__ int len_of(const wsr_attn& p, int b) { return min(max(p.lens[b], 0), (int)p.max_len); }

/* Row tile `tile` of `rows` rows over the sequences: its sequence, first row there, first token, rows of the
   sequence and its own keys. */
struct Place {
    int seq, row0, t0, rows, own;
};
__device__ __forceinline__ bool find_rows(const wsr_attn& p, int G, int rows, int tile, Place& o) {
    const int lane = threadIdx.x % WAVE;
    for (int b0 = 0; b0 < p.n_seqs; b0 += WAVE) {
        const int b = b0 + lane;
        int n = 0, first = 0, count = 0, len = 0;
        if (b < p.n_seqs) {
            first = start_of(p, b), len = len_of(p, b);
            count = max(start_of(p, b + 1) - first, 0) * G;
            n = (count + rows - 1) / rows;
        }
        int sum = n;                                            /* tiles up to and with this sequence */
#pragma unroll
        for (int k = 1; k < WAVE; k <<= 1) {
            const int v = __shfl_up(sum, k);
            if (lane >= k) sum += v;
        }
        const int all = __builtin_amdgcn_readlane(sum, WAVE - 1);
        if (tile < all) {
            const int w = __builtin_ctzll(__ballot(sum > tile));
            o.seq = b0 + w;
            o.row0 = (tile - (__builtin_amdgcn_readlane(sum, w) - __builtin_amdgcn_readlane(n, w))) * rows;
            o.t0 = __builtin_amdgcn_readlane(first, w), o.rows = __builtin_amdgcn_readlane(count, w);
            o.own = __builtin_amdgcn_readlane(len, w);
            return true;
        }
        tile -= all;
    }
    return false;
}

/* Row tiles over all sequences. */
__device__ __forceinline__ int count_tiles(const wsr_attn& p, int G, int rows) {
    int n = 0;
    for (int b = threadIdx.x % WAVE; b < p.n_seqs; b += WAVE) n += (max(start_of(p, b + 1) - start_of(p, b), 0) * G + rows - 1) / rows;
#pragma unroll
    for (int k = 32; k; k >>= 1) n += __shfl_xor(n, k);
    return __builtin_amdgcn_readfirstlane(n);
}

/* Keys of a part of a sequence's `own` keys (split form): of at most `parts` equal ones, whole blocks, LEAST or more
   where joining one costs less than the keys.  Taken from the length and not from the room that the cache has. */
constexpr int LEAST = 256;
__device__ __forceinline__ int own_part(int own, int parts, int block) {
    return (max(LEAST, (own - 1) / max(parts, 1) + 1) + block - 1) / block * block;
}

/* The units (row tile, key head) of the whole form: the first `full` go to a workgroup each, the other `rest` to
   `parts` of them each. */
constexpr int JOIN_ROWS = 4;
constexpr int HELD = 512;                      /* workgroups on the chip at a time: two per CU */
struct Round {
    int full, rest, parts;
};
__device__ __forceinline__ Round last_round(const wsr_attn& p, const AttnPlan& pl, int tiles) {
    const int units = tiles * p.n_kv_heads, rest = units % HELD, parts = rest ? min(pl.most_parts, HELD / rest) : 1;
    return parts > 1 ? Round{units - rest, rest, parts} : Round{units, 0, 1};
}

/* The blocks of keys that lie one after another, `stride` bytes from one key to the next. */
template <int FMT, int D, int RW>
struct Attend : AttendBlocks<FMT, D, RW> {
    typedef AttendBlocks<FMT, D, RW> B;
    using B::HALF, B::KS, B::DT, B::KT, B::KW, B::LOADS, B::PIECES, B::BUFFER, B::q, B::o, B::m, B::kswz, B::vswz, B::step;

    uint32_t koff[LOADS], voff[LOADS];                          /* a lane's places in a block in memory */

    /* A block of keys and values (rows k0 .. of kb, vb, those from k1 on replaced by the last before it) into a
       buffer of the group. */
    __device__ __forceinline__ void fetch(const char* kb, const char* vb, int64_t stride, int k0, int k1, l_char* buf, int rwave,
                                          int lane) const {
        const wsr::rsrc_t kr = wsr::buffer_of(kb + k0 * stride), vr = wsr::buffer_of(vb + k0 * stride);
        const int most = min(KT, k1 - k0) - 1;
        if (most == KT - 1) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int at = (rwave * LOADS + i) * WAVE;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, buf + at * 16, 16, koff[i], 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, buf + (HALF + at) * 16, 16, voff[i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int at = (rwave * LOADS + i) * WAVE, key = (at + lane) / PIECES, piece = (at + lane) % PIECES;
                const uint32_t row = (uint32_t)min(key, most) * (uint32_t)stride;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, buf + at * 16, 16, row + 16 * (piece ^ kswz(key)), 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, buf + (HALF + at) * 16, 16, row + 16 * (piece ^ vswz(key)), 0, 0, 0);
            }
        }
    }

    /* Blocks alternate between two buffers: a block is fetched while the one before it is worked on.  A wave with
       buffers of its own needs no barrier and fetches a block before it waits for the one before it, so that two
       are in flight (one token on 32771 keys, 32 heads on 8: 45 us with barriers, 37 without; groups of two or
       four waves, which would need a second barrier for it, gained nothing: 96 and 103 us, 59 and 60).
       The two pointers are declared not to alias, so that the compiler does not wait for the loads into `next`
       before it reads `cur`. */
    static constexpr bool DEEP = RW == 1;
    __device__ __forceinline__ void round(const l_char* __restrict cur, l_char* __restrict next, uint32_t group_at, const char* kb,
                                          const char* vb, int64_t stride, int at, int k1, int lim, int low, int high, float c,
                                          int rwave, int lane) {
        const bool more = at + KW * KT < k1;
        if constexpr (!DEEP) {
            wait_loads<0>();
            __syncthreads();                                    /* `cur` is there, `next` has been read */
            if (more) fetch(kb, vb, stride, at + KW * KT, k1, next + group_at, rwave, lane);
        } else if (more) {
            fetch(kb, vb, stride, at + KW * KT, k1, next + group_at, rwave, lane);
            wait_loads<2 * LOADS>();
        } else wait_loads<0>();
        const int end = min(at + KT, k1);
        if (at < min(end, high)) step(cur, min(lim, end) - at, min(low, end) < at + KT, c, lane);
    }

    /* Keys k0 .. k1 - 1; this lane's row sees those before `lim`, all rows of the wave those before `low`
       and none from `high` on.  Every wave of the workgroup takes part. */
    __device__ __forceinline__ void walk(const char* kb, const char* vb, int64_t stride, int k0, int k1, int lim, int low,
                                         int high, float c, l_char* lds, int wave, int lane) {
        const int rwave = wave % RW, group = wave / RW;
        const uint32_t group_at = group * 2 * BUFFER;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = (rwave * LOADS + i) * WAVE, key = (at + lane) / PIECES, piece = (at + lane) % PIECES;
            koff[i] = (uint32_t)key * (uint32_t)stride + 16 * (piece ^ kswz(key));
            voff[i] = (uint32_t)key * (uint32_t)stride + 16 * (piece ^ vswz(key));
        }
        int at = k0 + group * KT;
        if (at < k1) fetch(kb, vb, stride, at, k1, lds + group_at, rwave, lane);
        for (int left = (k1 - k0 + KW * KT - 1) / (KW * KT); left > 0; left -= 2) {
            round(lds, lds + BUFFER, group_at, kb, vb, stride, at, k1, lim, low, high, c, rwave, lane);
            at += KW * KT;
            if (left == 1) break;
            round(lds + BUFFER, lds, group_at, kb, vb, stride, at, k1, lim, low, high, c, rwave, lane);
            at += KW * KT;
        }
        __syncthreads();
    }

    /* Adds keys from .. to - 1, those before lim for this lane's row. */
    __device__ __forceinline__ void again(const char* kb, const char* vb, int64_t stride, int from, int to, int lim, float c, int lane) {
        const int h = lane / 32;
        const float base = m == A_NEG_INF ? 0.f : m * c;
#pragma unroll 1
        for (int key = from; key < to; ++key) {
            const char *kr = kb + key * stride, *vr = vb + key * stride;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const u32x4 w = ((const u32x4*)kr)[2 * k + h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float a, b, x, y;
                    unpack2<FMT>(w[j], a, b);
                    unpack2<FMT>(q[k][j], x, y);
                    s = fmaf(a, x, fmaf(b, y, s));
                }
            }
            s = wsr::xchg_add<0>(s);
            const bool see = key < lim;
            const float prob = see ? __builtin_amdgcn_exp2f(fmaf(s, c, -base)) : 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x2 w = *(const u32x2*)(vr + (32 * i + 8 * j + 4 * h) * 2);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float a, b;
                        unpack2<FMT>(see ? w[e] : 0u, a, b);
                        o[i][4 * j + 2 * e] = fmaf(prob, a, o[i][4 * j + 2 * e]);
                        o[i][4 * j + 2 * e + 1] = fmaf(prob, b, o[i][4 * j + 2 * e + 1]);
                    }
                }
        }
    }
};

/* The split form: workgroups below prefix_items take (key head, row tile, part) of the prefix, the others
   (key head, row tile, part) of a sequence's own keys; or, whole, both for a row tile of one sequence. */
template <int FMT, int D, int RW, bool WHOLE>
__global__ __launch_bounds__(AT) __attribute__((amdgpu_waves_per_eu(RW == 1 ? 1 : 2)))
void k_attn(wsr_attn p, AttnPlan pl) {
    typedef Attend<FMT, D, RW> A;
    __shared__ u32x4 lds[A::LDS];
    constexpr int ROWS = 32 * RW, BLOCK = A::KT * A::KW;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), rwave = wave % RW, col = lane % 32;
    const int G = p.n_heads / p.n_kv_heads;
    int item = blockIdx.x, part = 0, parts = 1;
    if (WHOLE) {
        const Round r = last_round(p, pl, count_tiles(p, G, ROWS));
        if (item >= r.full) {
            const int j = item - r.full;
            if (j >= r.rest * r.parts) return;
            part = j / r.rest, parts = r.parts, item = r.full + j % r.rest;
        }
    }
    const int head = item % p.n_kv_heads;
    item /= p.n_kv_heads;
    const bool prefix = !WHOLE && item < pl.prefix_tiles * pl.prefix_parts;
    int seq = 0, row0, t0 = 0, rows, own = 0;
    if (prefix) {
        row0 = item % pl.prefix_tiles * ROWS;
        part = item / pl.prefix_tiles;
        rows = p.n_tokens * G;
    } else {
        if (!WHOLE) {
            item -= pl.prefix_tiles * pl.prefix_parts;
            part = item / pl.own_tiles;
            item %= pl.own_tiles;
        }
        Place o;
        if (!find_rows(p, G, ROWS, item, o)) return;
        seq = o.seq, row0 = o.row0, t0 = o.t0, rows = o.rows, own = o.own;
    }
    const int shared = (int)p.prefix_len;
    /* rows of a sequence: row i of its n sees own keys before past + i */
    const int past = own - rows / G + 1;
    const int seen = max(0, past + min(row0 + ROWS - 1, rows - 1) / G);    /* own keys that a row of the workgroup sees */
    int k0 = 0, k1 = 0;
    if (!WHOLE) {
        const int keys = prefix ? pl.prefix_part : own_part(own, pl.own_parts, BLOCK), all = prefix ? shared : own;
        if ((int64_t)part * keys >= all) return;
        k0 = part * keys;
        k1 = all - k0 > keys ? k0 + keys : all;
    } else {                                   /* of the prefix and the own keys behind it */
        const int all = shared + seen, keys = ((all + parts - 1) / parts + A::KT - 1) / A::KT * A::KT;
        k0 = min(part * keys, all);
        k1 = all - k0 > keys ? k0 + keys : all;
    }
    const int row = row0 + rwave * 32 + col;                    /* this lane's row, both halves the same */
    const bool valid = row < rows;
    const int at_row = min(row, rows - 1) / G, tok = t0 + at_row, qh = head * G + min(row, rows - 1) - at_row * G;
    A a;
    a.init(wave / RW * 2 * A::BUFFER, lane);
    {
        const char* qr = (const char*)p.q + tok * p.q_tok_stride + qh * p.q_head_stride;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) a.q[k] = ((const u32x4*)qr)[2 * k + lane / 32];
    }
    const float c = p.scale * A_LOG2E;
    const bool busy = row0 + rwave * 32 < rows;                 /* the wave has rows */
    /* the prefix, then the sequence's own keys: one copy of the loop for both */
#pragma unroll 1
    for (int s = WHOLE ? 0 : !prefix; s <= (WHOLE ? 1 : !prefix); ++s) {
        const int low = s ? past + min(row0 + rwave * 32, rows - 1) / G : k1;
        const int high = !busy ? 0 : s ? past + min(row0 + rwave * 32 + 31, rows - 1) / G : k1;
        const int b = WHOLE && s ? max(k0 - shared, 0) : k0;
        const int e = !s ? min(k1, shared) : WHOLE ? k1 - shared : min(k1, seen);
        if (e <= b) continue;
        const int64_t at = s ? seq * p.kv_seq_stride + head * p.kv_head_stride : head * p.prefix_head_stride;
        a.walk((const char*)(s ? p.k : p.k_prefix) + at, (const char*)(s ? p.v : p.v_prefix) + at,
               s ? p.kv_tok_stride : p.prefix_tok_stride, b, e, s ? past + at_row : k1, low, high, c, (l_char*)lds, wave, lane);
    }
    a.join(lds, c, wave, lane);
    if (wave >= RW) return;
    const bool mine = a.broken() && a.l == a.l;                 /* a NaN sum makes all of the row NaN as it is */
    if (__ballot(mine) && (!prefix || (k1 - k0) % A::KT)) {
        if (mine) a.clear();
#pragma unroll 1
        for (int s = WHOLE ? 0 : !prefix; s <= (WHOLE ? 1 : !prefix); ++s) {
            const int64_t at = s ? seq * p.kv_seq_stride + head * p.kv_head_stride : head * p.prefix_head_stride;
            const int b = WHOLE && s ? max(k0 - shared, 0) : k0, e = !s ? min(k1, shared) : WHOLE ? k1 - shared : min(k1, seen);
            a.again((const char*)(s ? p.k : p.k_prefix) + at, (const char*)(s ? p.v : p.v_prefix) + at,
                    s ? p.kv_tok_stride : p.prefix_tok_stride, b, e, !mine ? b : s ? past + at_row : e, c, lane);
        }
    }
    if (!valid) return;
    const int h = lane / 32;
    if (WHOLE && parts == 1) {
        const float inv = a.l > 0.f ? 1.f / a.l : a.l == 0.f ? 0.f : a.l;
        char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
#pragma unroll
        for (int i = 0; i < A::DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(u32x2*)(out + (32 * i + 8 * j + 4 * h) * 2) =
                    u32x2{pack2<FMT>(a.o[i][4 * j] * inv, a.o[i][4 * j + 1] * inv),
                          pack2<FMT>(a.o[i][4 * j + 2] * inv, a.o[i][4 * j + 3] * inv)};
        if (p.lse && h == 0) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(a.m, a.l, p.scale);
    } else {
        const int64_t slot = WHOLE ? (int64_t)(blockIdx.x % HELD) * ROWS + row - row0  /* full is a multiple of HELD */
                                   : ((int64_t)(prefix ? part : pl.prefix_parts + part) * p.n_tokens + tok) * p.n_heads + qh;
        float* w = pl.part + slot * (D + 4);
#pragma unroll
        for (int i = 0; i < A::DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(f4_t*)(w + 32 * i + 8 * j + 4 * h) =
                    f4_t{a.o[i][4 * j], a.o[i][4 * j + 1], a.o[i][4 * j + 2], a.o[i][4 * j + 3]};
        if (h == 0) w[D] = a.m, w[D + 1] = a.l;
    }
}

/* Adds up the n parts of a row, `step` floats apart, and stores it, by one wave: in order, AHEAD: eight, four, two and
   one of them loaded at a time (one by one, each after the one before has come, a token on 32771 keys took 36 us, so
   30.5; in the whole form, where many waves wait beside one another, one by one is 2 to 3 us of 354 to 389 faster). */
template <int FMT, int D, bool AHEAD>
__device__ __forceinline__ void join_row(const wsr_attn& p, const float* w, int64_t step, int n, int tok, int qh, int lane) {
    constexpr int E = D / WAVE;
    const float c = p.scale * A_LOG2E;
    float m = A_NEG_INF, l = 0.f, o[E] = {};
    auto add = [&](auto count) __attribute__((always_inline)) {
        constexpr int N = decltype(count)::value;
        float pm[N], ps[N], po[N][E];
#pragma unroll
        for (int k = 0; k < N; ++k, w += step) {
            pm[k] = w[D], ps[k] = w[D + 1];
#pragma unroll
            for (int e = 0; e < E; ++e) po[k][e] = w[E * lane + e];
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float top = fmaxf(m, pm[k]), base = top == A_NEG_INF ? 0.f : top * c;
            const float a = __builtin_amdgcn_exp2f(m * c - base), b = __builtin_amdgcn_exp2f(pm[k] * c - base);
            l = l * a + ps[k] * b;
            m = top;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * a + po[k][e] * b;
        }
    };
    if constexpr (AHEAD) {
        for (; n >= 8; n -= 8) add(std::integral_constant<int, 8>{});
        if (n & 4) add(std::integral_constant<int, 4>{});
        if (n & 2) add(std::integral_constant<int, 2>{});
        if (n & 1) add(std::integral_constant<int, 1>{});
    } else
        for (; n > 0; --n) add(std::integral_constant<int, 1>{});
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
    if constexpr (E == 2) ((uint32_t*)out)[lane] = pack2<FMT>(o[0] * inv, o[1] * inv);
    else ((uint16_t*)out)[lane] = (uint16_t)pack2<FMT>(o[0] * inv, 0.f);
    if (p.lse && lane == 0) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(m, l, p.scale);
}

/* One wave per (token, head), from row `first` on: the parts that were written, in order. */
template <int FMT, int D>
__global__ __launch_bounds__(AT) void k_attn_join(wsr_attn p, AttnPlan pl, int64_t first) {
    const int64_t row = first + (int64_t)blockIdx.x * AW + wsr::wave_in_block();
    const int lane = threadIdx.x % WAVE;
    if (row >= (int64_t)p.n_tokens * p.n_heads) return;
    const int tok = (int)(row / p.n_heads), qh = (int)(row % p.n_heads);
    /* the token's sequence: the last that starts at or before it */
    int seq = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += WAVE) {
        const int b = b0 + lane;
        const uint64_t in = __ballot(b < p.n_seqs && start_of(p, b) <= tok);
        seq += __builtin_popcountll(in);
    }
    seq = __builtin_amdgcn_readfirstlane(seq) - 1;
    int own = 0;
    if (seq >= 0 && tok < start_of(p, seq + 1)) {
        /* own keys that the token sees */
        const int seen = len_of(p, seq) - (start_of(p, seq + 1) - tok) + 1;
        if (seen > 0) own = (seen - 1) / own_part(len_of(p, seq), pl.own_parts, pl.own_block) + 1;
    }
    join_row<FMT, D, true>(p, pl.part + row * (D + 4), (int64_t)p.n_tokens * p.n_heads * (D + 4), pl.prefix_parts + own, tok, qh, lane);
}

/* The parts of the whole form's last round: a wave per row of its units. */
template <int FMT, int D>
__global__ __launch_bounds__(AT) void k_attn_join_units(wsr_attn p, AttnPlan pl) {
    constexpr int ROWS = 128;
    const int G = p.n_heads / p.n_kv_heads, lane = threadIdx.x % WAVE, wave = wsr::wave_in_block();
    const Round r = last_round(p, pl, count_tiles(p, G, ROWS));
    for (int i = blockIdx.x; i < r.rest * (ROWS / JOIN_ROWS); i += gridDim.x) {
        const int unit = i / (ROWS / JOIN_ROWS), item = r.full + unit;
        Place o;
        if (!find_rows(p, G, ROWS, item / p.n_kv_heads, o)) return;
        for (int k = wave; k < JOIN_ROWS; k += AW) {
            const int at = i % (ROWS / JOIN_ROWS) * JOIN_ROWS + k, row = o.row0 + at;
            if (row < o.rows)
                join_row<FMT, D, false>(p, pl.part + ((int64_t)unit * ROWS + at) * (D + 4), (int64_t)r.rest * ROWS * (D + 4), r.parts,
                                 o.t0 + row / G, item % p.n_kv_heads * G + row % G, lane);
        }
    }
}

/* ---- host ------------------------------------------------------------------------------------------ */

static int row_waves(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

static AttnPlan attn_plan(const wsr_attn& p) {
    AttnPlan pl{};
    const int64_t G = p.n_heads / p.n_kv_heads, rows = p.n_tokens * G;
    const int rw = row_waves(rows);
    /* with fewer rows of a sequence most of its row tile would be empty, and with fewer tiles the split form's
       joining costs less (2 x 300 queries on 2001 keys, 32 heads on 8: 47 us whole, 43 split) */
    pl.whole = rw == 4 && rows >= 64 * (int64_t)p.n_seqs && p.n_kv_heads * (rows / 128) >= HELD / 2;
    pl.most_parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(16, (p.prefix_len + p.max_len) / 256));
    pl.own_tiles = (int32_t)(rows / (32 * rw) + std::min<int64_t>(p.n_seqs, p.n_tokens));
    if (pl.whole) return pl;
    const int64_t tiles = (rows + 32 * rw - 1) / (32 * rw), per = tiles * p.n_kv_heads;
    pl.prefix_tiles = (int32_t)tiles;
    const int64_t block = rw == 4 ? 64 : 32 * (4 / rw), held = rw == 1 ? HELD / 2 : HELD;
    auto parts = [&](int64_t keys, int64_t units, int32_t& part) {
        if (keys <= 0) return (int32_t)0;
        const int64_t want = std::max<int64_t>(1, held / std::max<int64_t>(1, units));
        part = (int32_t)std::min<int64_t>((std::max<int64_t>(LEAST, (keys + want - 1) / want) + block - 1) / block * block, 1 << 30);
        return (int32_t)((keys + part - 1) / part);
    };
    int32_t longest;
    pl.prefix_parts = parts(p.prefix_len, per, pl.prefix_part);
    /* own_tiles is what there can be at most and sequences differ in length: parts for twice the places (41 sequences of
       9 queries 34.0 us, so 32.9; 17 of one 40.8 and 39.9; the prefix's, which are alike, would lose a fifth) */
    pl.own_parts = parts(p.max_len, ((int64_t)pl.own_tiles * p.n_kv_heads + 1) / 2, longest);
    pl.own_block = (int32_t)block;
    return pl;
}

/* Workgroups of the first launch. */
static int64_t attn_blocks(const wsr_attn& p, const AttnPlan& pl) {
    const int64_t items = pl.whole ? pl.own_tiles : (int64_t)pl.prefix_tiles * pl.prefix_parts + (int64_t)pl.own_tiles * pl.own_parts;
    return items * p.n_kv_heads + (pl.whole && pl.most_parts > 1 ? HELD : 0);
}
bool attn_fits(const wsr_attn& p) { return attn_blocks(p, attn_plan(p)) <= most_blocks(AT); }

size_t attn_workspace(const wsr_attn& p) {
    const AttnPlan pl = attn_plan(p);
    if (pl.whole) return pl.most_parts > 1 ? (size_t)HELD * 128 * (p.head_dim + 4) * 4 : 256;
    return std::max<size_t>(256, (size_t)(pl.prefix_parts + pl.own_parts) * p.n_tokens * p.n_heads * (p.head_dim + 4) * 4);
}

template <int FMT, int D>
static hipError_t launch_dim(const wsr_attn& p, const AttnPlan& pl, hipStream_t s) {
    const int64_t blocks = attn_blocks(p, pl);
    const dim3 grid((unsigned)blocks), threads(AT);
    if (blocks > 0) {
        if (pl.whole) hipLaunchKernelGGL((k_attn<FMT, D, 4, true>), grid, threads, 0, s, p, pl);
        else switch (row_waves((int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads))) {
            case 1: hipLaunchKernelGGL((k_attn<FMT, D, 1, false>), grid, threads, 0, s, p, pl); break;
            case 2: hipLaunchKernelGGL((k_attn<FMT, D, 2, false>), grid, threads, 0, s, p, pl); break;
            default: hipLaunchKernelGGL((k_attn<FMT, D, 4, false>), grid, threads, 0, s, p, pl); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || (pl.whole && pl.most_parts == 1)) return e;
    }
    if (pl.whole) {
        hipLaunchKernelGGL((k_attn_join_units<FMT, D>), dim3(2048), threads, 0, s, p, pl);
        return hipGetLastError();
    }
    const int64_t rows = (int64_t)p.n_tokens * p.n_heads;
    for (int64_t first = 0; first < rows; first += most_blocks(AT) * AW) {
        const int64_t n = std::min((rows - first + AW - 1) / AW, most_blocks(AT));
        hipLaunchKernelGGL((k_attn_join<FMT, D>), dim3((unsigned)n), threads, 0, s, p, pl, first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_attn(const wsr_attn& p, void* ws, hipStream_t s) {
    AttnPlan pl = attn_plan(p);
    pl.part = static_cast<float*>(ws);
    if (p.fmt == WSR_F16) return p.head_dim == 64 ? launch_dim<WSR_F16, 64>(p, pl, s) : launch_dim<WSR_F16, 128>(p, pl, s);
    return p.head_dim == 64 ? launch_dim<WSR_BF16, 64>(p, pl, s) : launch_dim<WSR_BF16, 128>(p, pl, s);
}

}  // namespace wsr_step
