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
 * Keys and values go from memory straight into LDS, two buffers, the next block in flight while one is
 * worked on; 16-byte pieces are placed so that reads meet no bank twice.
 *
 *  - split form (few rows): workgroups over parts of the prefix for all rows, and over parts of each
 *    sequence's own keys; each leaves a maximum, a sum and an unnormalised fp32 row, which
 *    k_attn_join adds up.
 *  - whole form (prompts): a workgroup takes 128 rows of one sequence through the prefix and its own
 *    keys and stores the result.
 */
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int AT = 256, AW = AT / WAVE;
constexpr float A_NEG_INF = -__builtin_inff();
constexpr float A_LOG2E = 1.4426950408889634f;

struct AttnPlan {
    int32_t prefix_tiles, prefix_parts;    /* row tiles and key parts of the prefix (split form) */
    int32_t own_tiles, own_parts;          /* most row tiles over all sequences, most key parts of one */
    int32_t prefix_part, own_part;         /* keys of a part */
    float* part;                           /* [(prefix_parts + own_parts)][n_tokens][n_heads][head_dim + 2] */
    bool whole;
};

/* The query tokens of sequence b. */
__device__ __forceinline__ int start_of(const wsr_attn& p, int b) {
    return p.starts ? min(max(p.starts[b], 0), p.n_tokens) : min(b, p.n_tokens);
}
__device__ __forceinline__ int len_of(const wsr_attn& p, int b) { return min(max(p.lens[b], 0), (int)p.max_len); }

/* Row tile `tile` of `rows` rows over the sequences: its sequence and its first row there. */
__device__ __forceinline__ bool find_rows(const wsr_attn& p, int G, int rows, int tile, int& seq, int& row0) {
    const int lane = threadIdx.x % WAVE;
    for (int b0 = 0; b0 < p.n_seqs; b0 += WAVE) {
        const int b = b0 + lane;
        int n = 0;
        if (b < p.n_seqs) n = (max(start_of(p, b + 1) - start_of(p, b), 0) * G + rows - 1) / rows;
        int sum = n;                                            /* tiles up to and with this sequence */
#pragma unroll
        for (int k = 1; k < WAVE; k <<= 1) {
            const int o = __shfl_up(sum, k);
            if (lane >= k) sum += o;
        }
        const int all = __shfl(sum, WAVE - 1);
        if (tile < all) {
            const uint64_t after = __ballot(sum > tile);
            const int w = __builtin_ctzll(after);
            seq = __builtin_amdgcn_readfirstlane(b0 + w);
            row0 = __builtin_amdgcn_readfirstlane((tile - (__shfl(sum, w) - __shfl(n, w))) * rows);
            return true;
        }
        tile -= all;
    }
    return false;
}

typedef __attribute__((address_space(3))) u32x4 l_u32x4;
typedef __attribute__((address_space(3))) char l_char;
typedef __attribute__((address_space(3))) s4_t l_s4;

/* The running maximum is only moved when a row's scores pass it by 2^LAZY: until then its probabilities are
   taken against the old one (at most 2^LAZY, exact after the division by their sum), and the sums and
   outputs need no rescaling. */
constexpr float LAZY = 8.f;

/* A workgroup's place: RW waves side by side over rows (32 each), KW = 4 / RW groups of them over
   alternate blocks of KT keys. */
template <int FMT, int D, int RW>
struct Attend {
    static constexpr int KW = AW / RW, KT = KW == 1 ? 64 : 32, TILES = KT / 32;
    static constexpr int PIECES = D / 8;                        /* 16-byte pieces of a key */
    static constexpr int ROW = 2 * D;                           /* bytes of a key */
    static constexpr int HALF = KT * PIECES;                    /* pieces of a block of keys (and of values) */
    static constexpr int BUFFER = 2 * HALF * 16;                /* bytes of one of a group's two buffers */
    static constexpr int LOADS = HALF / WAVE / RW;              /* of 64 pieces, per wave and plane */
    static constexpr int DT = D / 32, KS = D / 16;
    static constexpr int LDS = KW * 2 * 2 * HALF;               /* pieces of the workgroup */

    u32x4 q[KS];
    f16v_t o[DT];
    float m, l;                                                 /* the maximum that probabilities are taken against; this half's sum */
    uint32_t ka[KS], va[DT], koff[LOADS], voff[LOADS];          /* a lane's places in LDS and in a block in memory */

    /* Piece x of a key lies at x ^ swz: the 16 keys of a read of keys, and the four keys times four pieces of a
       transposing read of values, lie on the 64 banks once each (two keys of 64 share a round of banks). */
    static __device__ __forceinline__ int kswz(int key) { return D == 128 ? key & 15 : key >> 1 & 7; }
    static __device__ __forceinline__ int vswz(int key) {
        return D == 128 ? (key & 3) << 2 | (key >> 2 & 1) : (key >> 1 & 1) << 2 | (key >> 2 & 1);
    }

    /* Places relative to the first group's first buffer, `base` bytes on for the wave's own group. */
    __device__ __forceinline__ void init(uint32_t base, int lane) {
        const int col = lane % 32, h = lane / 32, r = lane % 16 / 4, c = 2 * (col / 16) + lane % 4 / 2;
#pragma unroll
        for (int k = 0; k < KS; ++k) ka[k] = base + col * ROW + ((2 * k + h) ^ kswz(col)) * 16;
#pragma unroll
        for (int i = 0; i < DT; ++i)
            va[i] = base + HALF * 16 + (4 * h + r) * ROW + ((4 * i + c) ^ vswz(4 * h + r)) * 16 + lane % 2 * 8;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
        m = A_NEG_INF, l = 0.f;
    }

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

    /* One block of keys in buffer `buf` (of the first group): `left` keys of it are visible to this lane's row. */
    __device__ __forceinline__ void step(const l_char* buf, int left, bool masked, float c, int lane) {
        const int h = lane / 32;
        f16v_t s[TILES];
        u32x4 kf[TILES][KS];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                kf[t][k] = *(const l_u32x4*)(buf + ka[k] + 32 * t * ROW);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[t][j] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) s[t] = mma_32x32x16<FMT>(kf[t][k], q[k], s[t]);
        }
        /* KS reads ahead of the products, then one read after each */
        __builtin_amdgcn_sched_group_barrier(0x100, KS, 0);
#pragma unroll
        for (int i = 0; i < (TILES - 1) * KS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, KS, 0);
        /* values of 16 keys at a time, the next 16 in flight */
        u32x4 vf[2][DT];
        auto values = [&](u32x4 (&f)[DT], int t, int k) {
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 w = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((l_s4*)(buf + va[i] + (32 * t + 16 * k + 8 * e) * ROW)));
                    f[i][2 * e] = w.x, f[i][2 * e + 1] = w.y;
                }
        };
        __builtin_amdgcn_sched_barrier(0);
        values(vf[0], 0, 0);
        if (masked) {
            asm volatile("");                                   /* a branch: without it every block pays for the selects */
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (32 * t + 8 * (j / 4) + 4 * h + j % 4 >= left) s[t][j] = A_NEG_INF;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[t][j]);
        top = fmaxf(top, __shfl_xor(top, 32));
        /* (top - m) c > LAZY, true too where m is -inf and top is not */
        if (__ballot((top - m) * c > LAZY)) {
            const float next = fmaxf(m, top), f = next == A_NEG_INF ? 1.f : __builtin_amdgcn_exp2f((m - next) * c);
            l *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= f;
            m = next;
        }
        const float base = m == A_NEG_INF ? 0.f : m * c;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[t][j] = __builtin_amdgcn_exp2f(fmaf(s[t][j], c, -base));
                l += s[t][j];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {                       /* 16 keys */
                if (t + 1 < TILES || k == 0) values(vf[(k + 1) & 1], k == 0 ? t : t + 1, (k + 1) & 1);
                u32x4 pt;
#pragma unroll
                for (int j = 0; j < 4; ++j) pt[j] = pack2<FMT>(s[t][8 * k + 2 * j], s[t][8 * k + 2 * j + 1]);
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = mma_32x32x16<FMT>(vf[k][i], pt, o[i]);
            }
        }
    }

    /* Fetches a block into `next` and works on the one in `cur`.  The two pointers are declared not to alias, so
       that the compiler does not wait for the loads into `next` before it reads `cur`. */
    __device__ __forceinline__ void round(const l_char* __restrict cur, l_char* __restrict next, uint32_t group_at, const char* kb,
                                          const char* vb, int64_t stride, int at, int k1, int lim, int low, int high, float c,
                                          int rwave, int lane) {
        if (at + KW * KT < k1) fetch(kb, vb, stride, at + KW * KT, k1, next + group_at, rwave, lane);
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
            wait_loads<0>();
            __syncthreads();                                    /* this block is in LDS, the one before is done with */
            round(lds, lds + BUFFER, group_at, kb, vb, stride, at, k1, lim, low, high, c, rwave, lane);
            at += KW * KT;
            if (left == 1) break;
            wait_loads<0>();
            __syncthreads();
            round(lds + BUFFER, lds, group_at, kb, vb, stride, at, k1, lim, low, high, c, rwave, lane);
            at += KW * KT;
        }
        __syncthreads();
    }

    /* Adds up the groups' results in LDS; the first group's waves hold the row's maximum, sum (both halves)
       and output afterwards. */
    __device__ __forceinline__ void join(u32x4* lds, float c, int wave, int lane) {
        l += __shfl_xor(l, 32);
        if constexpr (KW > 1) {
            float* f = (float*)lds;
            constexpr int PER = WAVE * (16 * DT + 2);           /* floats that a wave leaves */
            static_assert((AW - RW) * PER * 4 <= LDS * 16, "the waves' results fit the key buffers");
            if (wave >= RW) {
                float* w = f + (wave - RW) * PER + lane;
                w[0] = m, w[WAVE] = l;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[(2 + 16 * i + j) * WAVE] = o[i][j];
            }
            __syncthreads();
            if (wave < RW) {
#pragma unroll
                for (int g = 1; g < KW; ++g) {
                    const float* w = f + ((g - 1) * RW + wave) * PER + lane;
                    const float m2 = w[0], top = fmaxf(m, m2), base = top == A_NEG_INF ? 0.f : top * c;
                    const float a = __builtin_amdgcn_exp2f(m * c - base), b = __builtin_amdgcn_exp2f(m2 * c - base);
                    l = l * a + w[WAVE] * b;
                    m = top;
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[i][j] = o[i][j] * a + w[(2 + 16 * i + j) * WAVE] * b;
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
    constexpr int ROWS = 32 * RW;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), rwave = wave % RW, col = lane % 32;
    const int G = p.n_heads / p.n_kv_heads;
    const int head = blockIdx.x % p.n_kv_heads;
    int item = blockIdx.x / p.n_kv_heads;
    const bool prefix = !WHOLE && item < pl.prefix_tiles * pl.prefix_parts;
    int seq = 0, row0, part, t0 = 0, rows;
    if (prefix) {
        row0 = item % pl.prefix_tiles * ROWS;
        part = item / pl.prefix_tiles;
        rows = p.n_tokens * G;
    } else {
        if (!WHOLE) item -= pl.prefix_tiles * pl.prefix_parts;
        part = WHOLE ? 0 : item / pl.own_tiles;
        if (!find_rows(p, G, ROWS, WHOLE ? item : item % pl.own_tiles, seq, row0)) return;
        t0 = __builtin_amdgcn_readfirstlane(start_of(p, seq));
        rows = __builtin_amdgcn_readfirstlane((start_of(p, seq + 1) - t0) * G);
    }
    const int own = prefix ? 0 : __builtin_amdgcn_readfirstlane(len_of(p, seq)), shared = (int)p.prefix_len;
    int k0 = 0, k1 = 0;
    if (!WHOLE) {
        const int keys = prefix ? pl.prefix_part : pl.own_part, all = prefix ? shared : own;
        if ((int64_t)part * keys >= all) return;
        k0 = part * keys;
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
    if (WHOLE || prefix) {
        const int e = WHOLE ? shared : k1;
        if (e > k0)
            a.walk((const char*)p.k_prefix + head * p.prefix_head_stride, (const char*)p.v_prefix + head * p.prefix_head_stride,
                   p.prefix_tok_stride, k0, e, e, e, busy ? e : 0, c, (l_char*)lds, wave, lane);
    }
    if (WHOLE || !prefix) {
        /* row i of the sequence's n: keys before own - n + i + 1 */
        const int past = own - rows / G + 1;
        const int low = past + min(row0 + rwave * 32, rows - 1) / G;
        const int high = busy ? past + min(row0 + rwave * 32 + 31, rows - 1) / G : 0;
        const int e = min(WHOLE ? own : k1, past + min(row0 + ROWS - 1, rows - 1) / G);   /* of the workgroup's rows */
        if (e > k0)
            a.walk((const char*)p.k + seq * p.kv_seq_stride + head * p.kv_head_stride,
                   (const char*)p.v + seq * p.kv_seq_stride + head * p.kv_head_stride, p.kv_tok_stride, k0, e, past + at_row,
                   low, high, c, (l_char*)lds, wave, lane);
    }
    a.join(lds, c, wave, lane);
    if (wave >= RW || !valid) return;
    const int h = lane / 32;
    if (WHOLE) {
        const float inv = a.l > 0.f ? 1.f / a.l : a.l == 0.f ? 0.f : a.l;
        char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
#pragma unroll
        for (int i = 0; i < A::DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(u32x2*)(out + (32 * i + 8 * j + 4 * h) * 2) =
                    u32x2{pack2<FMT>(a.o[i][4 * j] * inv, a.o[i][4 * j + 1] * inv),
                          pack2<FMT>(a.o[i][4 * j + 2] * inv, a.o[i][4 * j + 3] * inv)};
        if (p.lse && h == 0) p.lse[(int64_t)tok * p.n_heads + qh] = a.m == A_NEG_INF ? a.m : a.m * p.scale + logf(a.l);
    } else {
        const int64_t slot = ((int64_t)(prefix ? part : pl.prefix_parts + part) * p.n_tokens + tok) * p.n_heads + qh;
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

/* One wave per (token, head): the parts that were written, in order. */
template <int FMT, int D>
__global__ __launch_bounds__(AT) void k_attn_join(wsr_attn p, AttnPlan pl) {
    const int64_t row = (int64_t)blockIdx.x * AW + wsr::wave_in_block();
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
        if (seen > 0) own = (seen - 1) / pl.own_part + 1;
    }
    const int n = pl.prefix_parts + own;
    constexpr int E = D / WAVE;
    const int64_t step = (int64_t)p.n_tokens * p.n_heads * (D + 4);
    const float* w = pl.part + row * (D + 4);
    const float c = p.scale * A_LOG2E;
    float m = A_NEG_INF, l = 0.f, o[E] = {};
    for (int i = 0; i < n; ++i) {
        const float* v = w + i * step;
        const float m2 = v[D], top = fmaxf(m, m2), base = top == A_NEG_INF ? 0.f : top * c;
        const float a = __builtin_amdgcn_exp2f(m * c - base), b = __builtin_amdgcn_exp2f(m2 * c - base);
        l = l * a + v[D + 1] * b;
        m = top;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * a + v[E * lane + e] * b;
    }
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
    if constexpr (E == 2) ((uint32_t*)out)[lane] = pack2<FMT>(o[0] * inv, o[1] * inv);
    else ((uint16_t*)out)[lane] = (uint16_t)pack2<FMT>(o[0] * inv, 0.f);
    if (p.lse && lane == 0) p.lse[row] = m == A_NEG_INF ? m : m * p.scale + logf(l);
}

/* ---- host ------------------------------------------------------------------------------------------ */

constexpr int64_t WHOLE_TILES = 256;           /* row tiles times key heads from which the whole form is taken */

static int row_waves(int64_t rows) { return rows <= 32 ? 1 : rows <= 64 ? 2 : 4; }

static AttnPlan attn_plan(const wsr_attn& p) {
    AttnPlan pl{};
    const int64_t G = p.n_heads / p.n_kv_heads, rows = p.n_tokens * G;
    const int rw = row_waves(rows);
    pl.whole = rw == 4 && p.n_kv_heads * (rows / 128) >= WHOLE_TILES && rows >= 64 * (int64_t)p.n_seqs;
    pl.own_tiles = (int32_t)(rows / (32 * rw) + std::min<int64_t>(p.n_seqs, p.n_tokens));
    if (pl.whole) return pl;
    const int64_t tiles = (rows + 32 * rw - 1) / (32 * rw), per = tiles * p.n_kv_heads;
    pl.prefix_tiles = (int32_t)tiles;
    const int64_t block = rw == 4 ? 64 : 64 * (4 / rw);
    auto parts = [&](int64_t keys, int64_t units, int64_t least, int32_t& part) {
        if (keys <= 0) return (int32_t)0;
        const int64_t want = std::max<int64_t>(1, 512 / std::max<int64_t>(1, units));
        part = (int32_t)std::min<int64_t>((std::max(least, (keys + want - 1) / want) + block - 1) / block * block, 1 << 30);
        return (int32_t)((keys + part - 1) / part);
    };
    pl.prefix_parts = parts(p.prefix_len, per, 256, pl.prefix_part);
    pl.own_parts = parts(p.max_len, (int64_t)pl.own_tiles * p.n_kv_heads, 256, pl.own_part);
    return pl;
}

size_t attn_workspace(const wsr_attn& p) {
    const AttnPlan pl = attn_plan(p);
    if (pl.whole) return 256;
    return std::max<size_t>(256, (size_t)(pl.prefix_parts + pl.own_parts) * p.n_tokens * p.n_heads * (p.head_dim + 4) * 4);
}

template <int FMT, int D>
static hipError_t launch_dim(const wsr_attn& p, const AttnPlan& pl, hipStream_t s) {
    const int64_t items = pl.whole ? pl.own_tiles : (int64_t)pl.prefix_tiles * pl.prefix_parts + (int64_t)pl.own_tiles * pl.own_parts;
    const int64_t blocks = items * p.n_kv_heads;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), threads(AT);
    if (blocks > 0) {
        if (pl.whole) hipLaunchKernelGGL((k_attn<FMT, D, 4, true>), grid, threads, 0, s, p, pl);
        else switch (row_waves((int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads))) {
            case 1: hipLaunchKernelGGL((k_attn<FMT, D, 1, false>), grid, threads, 0, s, p, pl); break;
            case 2: hipLaunchKernelGGL((k_attn<FMT, D, 2, false>), grid, threads, 0, s, p, pl); break;
            default: hipLaunchKernelGGL((k_attn<FMT, D, 4, false>), grid, threads, 0, s, p, pl); break;
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || pl.whole) return e;
    }
    const int64_t rows = (int64_t)p.n_tokens * p.n_heads;
    hipLaunchKernelGGL((k_attn_join<FMT, D>), dim3((unsigned)((rows + AW - 1) / AW)), threads, 0, s, p, pl);
    return hipGetLastError();
}

hipError_t launch_attn(const wsr_attn& p, void* ws, hipStream_t s) {
    AttnPlan pl = attn_plan(p);
    pl.part = static_cast<float*>(ws);
    if (p.fmt == WSR_F16) return p.head_dim == 64 ? launch_dim<WSR_F16, 64>(p, pl, s) : launch_dim<WSR_F16, 128>(p, pl, s);
    return p.head_dim == 64 ? launch_dim<WSR_BF16, 64>(p, pl, s) : launch_dim<WSR_BF16, 128>(p, pl, s);
}

}  // namespace wsr_step
