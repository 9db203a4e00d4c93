/*
 * wsr_paged.hip - attention of each sequence's newest tokens over its pages.
 *
 * A query row is one (token, query head); the rows of a sequence and key head, tokens times G = n_heads / n_kv_heads, go in
 * tiles of R.  The work of all tiles lies on one line, a tile as long as the keys it sees, and every workgroup takes an
 * equal share of that line, whatever the lengths on the device are: a share covers parts of one tile or many.  A tile that
 * lies in one share is stored at once; of the others each share leaves a maximum, a sum and an unnormalised fp32 row,
 * which k_paged_join adds up.
 *
 * A wave walks blocks of 32 keys with a running maximum and sum:
 *
 *   S^T = K Q^T   (v_mfma 16x16x32: 16 keys x 16 rows, each lane one row and four keys)
 *   P   = exp2((S - max) scale log2 e),  O^T += V^T P^T with P still in the registers of S: the lane layout of S^T is
 *         the operand layout of P^T when V's keys are taken in the same order
 *
 * Keys come from memory straight into operand layout (lane l: key l % 16, pieces l / 16, + 4, ..), since any order of a
 * head's dimensions gives the same product; values go through LDS, where transposing reads turn them.  The four waves of a
 * workgroup take blocks in turn and add up in LDS.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_serve_device.h"

namespace wsr_serve {

constexpr int AT = 256, AW = AT / WAVE;
constexpr int KT = 32;                        /* keys of a wave's block */
typedef short s4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char l_char;
typedef __attribute__((address_space(3))) u32x4 l_u32x4;
typedef __attribute__((address_space(3))) s4_t l_s4;
typedef __attribute__((address_space(3))) f4_t l_f4;
typedef __attribute__((address_space(3))) float l_float;

/* The running maximum is only moved when a row's scores pass it by 2^LAZY: until then its probabilities are taken
   against the old one (at most 2^LAZY, exact after the division by their sum). */
constexpr float LAZY = 8.f;

struct PagedPlan {
    int32_t rows;                             /* R, rows of a tile */
    int32_t shares;                           /* workgroups at most */
    uint64_t magic;                           /* division by page_size: (n * magic) >> shift for n < 2^31 */
    int32_t shift;
    float* part;                              /* [2 * shares][R][head_dim + 4] */
};

/* ---- the line of work ------------------------------------------------------------------------------

   Tile t of a sequence (of T, rows R t .. to its last) costs, per key head, past G + min(R (t + 1), rows) + A: G times the
   keys that its last row sees, and A for the tile itself.  Lengths on the line are at most 2^62 (2^26 rows in all, G at
   most 2^9, places below 2^31). */
struct Seq {
    int32_t t0, n, len;                       /* first token, tokens, keys */
    int32_t rows, tiles;
    int64_t flat, cost;                       /* past G + A; all tiles of a key head */
};
constexpr int EXTRA = 64;                     /* A, in keys */

__device__ __forceinline__ Seq seq_at(const wsr_paged& p, int R, int b) {
    Seq s;
    const int G = p.n_heads / p.n_kv_heads;
    int next;
    if (p.starts) {
        s.t0 = min(max(p.starts[b], 0), p.n_tokens);
        next = min(max(p.starts[b + 1], s.t0), p.n_tokens);
    } else s.t0 = b, next = b + 1;
    s.n = next - s.t0;
    s.len = (int)min(max((int64_t)p.lens[b], (int64_t)0), p.max_len);
    s.rows = s.n * G;
    s.tiles = (s.rows + R - 1) / R;
    s.flat = (int64_t)(max(s.len - s.n, 0) + EXTRA) * G;
    s.cost = s.tiles ? s.tiles * s.flat + (int64_t)R * s.tiles * (s.tiles - 1) / 2 + s.rows : 0;
    return s;
}
__device__ __forceinline__ int64_t before_tile(const Seq& s, int R, int t) { return t * s.flat + (int64_t)R * t * (t + 1) / 2; }
__device__ __forceinline__ int64_t tile_cost(const Seq& s, int R, int t) { return s.flat + min((int64_t)R * (t + 1), (int64_t)s.rows); }

__device__ __forceinline__ int64_t lane64(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}
/* The lanes' sums of themselves and those below. */
__device__ __forceinline__ int64_t scan64(int64_t v, int lane) {
#pragma unroll
    for (int k = 1; k < WAVE; k <<= 1) {
        const int64_t o = __shfl_up((long long)v, k);
        if (lane >= k) v += o;
    }
    return v;
}
/* Costs of the sequences before b0 + the lane's own and with it, given those before b0. */
__device__ __forceinline__ int64_t costs_to(const wsr_paged& p, int R, int b0, int64_t before, int lane) {
    return before + scan64(b0 + lane < p.n_seqs ? seq_at(p, R, b0 + lane).cost * p.n_kv_heads : 0, lane);
}

/* The line cut into shares: share w starts at w / shares of it. */
struct Line {
    int64_t all, each, rest;                  /* its length; all / shares, all % shares */
    int32_t shares;
    __device__ __forceinline__ int64_t start(int w) const { return each * w + rest * w / shares; }
    __device__ __forceinline__ int share_of(int64_t x) const {
        int w = min((int)((double)x / (double)all * shares), shares - 1);
        while (w > 0 && start(w) > x) --w;
        while (w + 1 < shares && start(w + 1) <= x) ++w;
        return w;
    }
};
constexpr int LEAST = 256;                    /* keys of a share at least */

__device__ __forceinline__ Line line_of(const wsr_paged& p, const PagedPlan& pl, int lane) {
    Line l;
    l.all = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += WAVE) l.all = lane64(costs_to(p, pl.rows, b0, l.all, lane), WAVE - 1);
    const int64_t least = (int64_t)(p.n_heads / p.n_kv_heads) * (LEAST + EXTRA);
    l.shares = (int)min((int64_t)pl.shares, max((l.all + least - 1) / least, (int64_t)1));
    l.each = l.all / l.shares, l.rest = l.all % l.shares;
    return l;
}

/* Keys of a tile up to offset o of its cost, in whole blocks; all `seen` from the end of the cost on. */
__device__ __forceinline__ int keys_to(int64_t o, int64_t cost, int seen, int G, int block) {
    if (o <= 0) return 0;
    if (o >= cost) return seen;
    return (int)min((int64_t)((double)o / ((double)G * block)) * block, (int64_t)seen);
}

/* ---- a wave's walk ----------------------------------------------------------------------------------- */

template <int FMT, int D, int RT>             /* RT: tiles of 16 rows */
struct Walk {
    static constexpr int KS = D / 32, DT = D / 16, PIECES = D / 8, ROW = 2 * D, R = 16 * RT;
    static constexpr int BUFFER = KT * ROW;                     /* bytes of a wave's values in LDS */
    static constexpr int SUMS = WAVE * (DT + 1) * 16;           /* bytes of a wave's results in LDS, of one tile */
    static constexpr int LDS = AW * (BUFFER > SUMS ? BUFFER : SUMS);

    u32x4 q[RT][KS];
    f4_t o[RT][DT];
    float m[RT], l[RT];
    u32x4 k[2][KS], v[2][KS];                                   /* keys and values: key l % 16 of each half, pieces l / 16 + 4 i */
    int entry[2], slot[2];                                      /* of the next block */
    uint32_t there;                                             /* keys of the loaded block that are on a page */

    static __device__ __forceinline__ int swz(int key) { return ((key & 3) << 2 | (key >> 2 & 3)) & (PIECES - 1); }

    __device__ __forceinline__ void look_up(const wsr_pages& c, const PagedPlan& pl, const int32_t* table, int at, int k1, int lane) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int key = min(at + 16 * h + lane % 16, k1 - 1);
            const int page = (int)((uint64_t)key * pl.magic >> pl.shift);
            slot[h] = key - page * c.page_size;
            entry[h] = table[page];
        }
    }
    __device__ __forceinline__ void load(const wsr_pages& c, const char* kb, const char* vb, int at, int k1, int lane) {
        int64_t off[2];
        uint64_t ok[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            ok[h] = __ballot((uint32_t)entry[h] < (uint32_t)c.n_pages && at + 16 * h + lane % 16 < k1);
            off[h] = entry[h] * c.page_stride + slot[h] * c.tok_stride;
        }
        there = (uint32_t)(ok[0] & 0xffff) | (uint32_t)(ok[1] & 0xffff) << 16;
        if (!there) return;
        if (there != 0xffffffffu) {                             /* the others repeat the first that is there */
            const int f = __builtin_ctz(there);
            const int64_t first = lane64(f < 16 ? off[0] : off[1], f % 16);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (!(there >> (16 * h + lane % 16) & 1)) off[h] = first;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < KS; ++i) k[h][i] = ((const u32x4*)(kb + off[h]))[4 * i + lane / 16];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < KS; ++i) v[h][i] = ((const u32x4*)(vb + off[h]))[4 * i + lane / 16];
    }

    /* The loaded block, keys at .. + 31, of which this lane's rows see those before lim; `all` where every row sees every key. */
    __device__ __forceinline__ void scores(f4_t (&s)[RT][2]) const {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[t][h] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) s[t][h] = wsr_step::mma16<FMT>(k[h][i], q[t][i], s[t][h]);
            }
    }
    __device__ __forceinline__ void keep_values(l_char* buf, int lane) const {
        const int key = lane % 16;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < KS; ++i)
                *(l_u32x4*)(buf + (16 * h + key) * ROW + ((4 * i + lane / 16) ^ swz(key)) * 16) = v[h][i];
    }
    __device__ __forceinline__ void weigh(f4_t (&s)[RT][2], uint32_t seen, bool masked, const int (&lim)[RT], int at, float c,
                                          const l_char* buf, int lane) {
        const int g = lane / 16;
        u32x4 pt[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            if (masked) {
                asm volatile("");                               /* a branch: without it every block pays for the selects */
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = 16 * h + 4 * g + j;
                        if (!(seen >> key & 1) || at + key >= lim[t]) s[t][h][j] = NEG_INF;
                    }
            }
            float top = s[t][0][0];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, s[t][h][j]);
            top = wsr_step::xchg_max<1>(wsr_step::xchg_max<0>(top));
            /* (top - m) c > LAZY, true too where m is -inf and top is not */
            if (__ballot((top - m[t]) * c > LAZY)) {
                const float next = fmaxf(m[t], top), f = next == NEG_INF ? 1.f : __builtin_amdgcn_exp2f((m[t] - next) * c);
                l[t] *= f;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[t][i][j] *= f;
                m[t] = next;
            }
            const float base = m[t] == NEG_INF ? 0.f : m[t] * c;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[t][h][j] = __builtin_amdgcn_exp2f(fmaf(s[t][h][j], c, -base));
                    l[t] += s[t][h][j];
                }
                pt[t][2 * h] = pack2<FMT>(s[t][h][0], s[t][h][1]);
                pt[t][2 * h + 1] = pack2<FMT>(s[t][h][2], s[t][h][3]);
            }
        }
        const int key = 4 * g + lane % 16 / 4;                  /* the lane's part of a transposing read */
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            u32x4 f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 w = __builtin_bit_cast(
                    u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                               (l_s4*)(buf + (16 * h + key) * ROW + ((2 * i + lane % 4 / 2) ^ swz(key)) * 16 + lane % 2 * 8)));
                f[2 * h] = w.x, f[2 * h + 1] = w.y;
            }
#pragma unroll
            for (int t = 0; t < RT; ++t) o[t][i] = wsr_step::mma16<FMT>(f, pt[t], o[t][i]);
        }
    }

    /* The products take keys that a row does not see with a probability of zero, and zero times an infinity or NaN among
       their values would reach it.  Such a row is found by its output and summed up again, key by key over those it sees,
       against the maximum it has: nothing is paid for it in the loop. */
    __device__ __forceinline__ bool broken(int t) const {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) z = fmaf(o[t][i][j], 0.f, z);
        z = wsr::xchg_add<1>(wsr::xchg_add<0>(z));
        return z != z;
    }
    __device__ __forceinline__ void again(int t, bool mine, const wsr_pages& c, const int32_t* table, const char* kb, const char* vb,
                                          int from, int to, int lim, float scale, int lane) {
        const int g = lane / 16;
        const float base = m[t] == NEG_INF ? 0.f : m[t] * scale;
#pragma unroll 1
        for (int key = from; key < to; ++key) {
            const int page = key / c.page_size, at = table[page];
            if ((uint32_t)at >= (uint32_t)c.n_pages) continue;
            const int64_t off = at * c.page_stride + (key - page * c.page_size) * c.tok_stride;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const u32x4 w = ((const u32x4*)(kb + off))[4 * i + g];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float a, b, x, y;
                    unpack2<FMT>(w[j], a, b);
                    unpack2<FMT>(q[t][i][j], x, y);
                    s = fmaf(a, x, fmaf(b, y, s));
                }
            }
            s = wsr::xchg_add<1>(wsr::xchg_add<0>(s));
            const bool see = mine && key < lim;
            const float prob = see ? __builtin_amdgcn_exp2f(fmaf(s, scale, -base)) : 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const u32x2 w = *(const u32x2*)(vb + off + (16 * i + 4 * g) * 2);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float a, b;
                    unpack2<FMT>(see ? w[j] : 0u, a, b);
                    o[t][i][2 * j] = fmaf(prob, a, o[t][i][2 * j]);
                    o[t][i][2 * j + 1] = fmaf(prob, b, o[t][i][2 * j + 1]);
                }
            }
        }
    }
};

/* log of a row's sum l against its maximum m: -inf where it saw no key, NaN where a score was. */
__device__ __forceinline__ float lse_of(float m, float l, float scale) { return l == 0.f ? NEG_INF : m * scale + logf(l); }
__device__ __forceinline__ float inverse_of(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; }

template <int FMT, int D, int RT>
__global__ __launch_bounds__(AT) void k_paged(wsr_paged p, PagedPlan pl) {
    typedef Walk<FMT, D, RT> W;
    constexpr int R = W::R;
    __shared__ u32x4 lds_room[W::LDS / 16];
    l_char* lds = (l_char*)lds_room;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    const int G = p.n_heads / p.n_kv_heads, N = p.n_kv_heads;
    const float c = p.scale * LOG2E;
    const Line line = line_of(p, pl, lane);
    const int share = blockIdx.x;
    if (share >= line.shares) return;
    const int64_t start = line.start(share);
    int64_t left = line.start(share + 1) - start;
    if (left <= 0) return;
    /* the place on the line: sequence, key head, tile, and how far into it */
    int b = 0;
    int64_t before = 0;
    for (int b0 = 0; b0 < p.n_seqs; b0 += WAVE) {
        const int64_t to = costs_to(p, R, b0, before, lane);
        const uint64_t past = __ballot(to > start);
        if (past) {
            const int w = __builtin_ctzll(past);
            b = b0 + w;
            if (w) before = lane64(to, w - 1);
            break;
        }
        before = lane64(to, WAVE - 1);
    }
    Seq s = seq_at(p, R, b);
    if (s.cost <= 0) return;
    int64_t o = start - before;
    int head = min((int)((double)o / (double)s.cost), N - 1);
    while (head > 0 && head * s.cost > o) --head;
    while (head + 1 < N && (head + 1) * s.cost <= o) ++head;
    o -= head * s.cost;
    int tile = 0;
    for (int lo = 0, hi = s.tiles; lo < hi;) {                   /* the last that starts at or before o */
        const int mid = (lo + hi) / 2;
        if (before_tile(s, R, mid) <= o) tile = mid, lo = mid + 1;
        else hi = mid;
    }
    o -= before_tile(s, R, tile);

    W w;
#pragma unroll 1
    while (true) {
        const int64_t cost = tile_cost(s, R, tile), take = min(left, cost - o);
        const int row0 = tile * R, last = min(row0 + R, s.rows) - 1, past = s.len - s.n;
        const int seen = max(past + last / G + 1, 0);
        const int k0 = keys_to(o, cost, seen, G, KT * AW), k1 = keys_to(o + take, cost, seen, G, KT * AW);
        const bool whole = take == cost;
        const char* kb = (const char*)p.cache.k + head * p.cache.head_stride;
        const char* vb = (const char*)p.cache.v + head * p.cache.head_stride;
        const int32_t* table = (const int32_t*)((const char*)p.cache.table + b * p.cache.table_stride);
        int lim[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const int row = min(row0 + 16 * t + col, last), at = row / G;
            lim[t] = past + at + 1;
            const char* qr = (const char*)p.q + (s.t0 + at) * p.q_tok_stride + (head * G + row - at * G) * p.q_head_stride;
#pragma unroll
            for (int i = 0; i < W::KS; ++i) w.q[t][i] = ((const u32x4*)qr)[4 * i + g];
#pragma unroll
            for (int i = 0; i < W::DT; ++i) w.o[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
            w.m[t] = NEG_INF, w.l[t] = 0.f;
        }
        const int all = past + row0 / G + 1;                    /* keys that every row sees */
        l_char* buf = lds + wave * W::BUFFER;
        int at = k0 + wave * KT;
        if (at < k1) {
            w.look_up(p.cache, pl, table, at, k1, lane);
            w.load(p.cache, kb, vb, at, k1, lane);
            if (at + AW * KT < k1) w.look_up(p.cache, pl, table, at + AW * KT, k1, lane);
        }
#pragma unroll 1
        for (; at < k1; at += AW * KT) {
            const uint32_t there = w.there;
            f4_t sc[RT][2];
            if (there) {
                w.scores(sc);
                w.keep_values(buf, lane);
            }
            if (at + AW * KT < k1) {
                w.load(p.cache, kb, vb, at + AW * KT, k1, lane);
                if (at + 2 * AW * KT < k1) w.look_up(p.cache, pl, table, at + 2 * AW * KT, k1, lane);
            }
            if (there) w.weigh(sc, there, there != 0xffffffffu || at + KT > all, lim, at, c, buf, lane);
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            w.l[t] = wsr::xchg_add<1>(wsr::xchg_add<0>(w.l[t]));
            const bool mine = w.broken(t) && w.l[t] == w.l[t];  /* a NaN sum makes all of the row NaN as it is */
            if (__ballot(mine)) {
                if (mine)
#pragma unroll
                    for (int i = 0; i < W::DT; ++i) w.o[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int k = k0 + wave * KT; k < k1; k += AW * KT)
                    w.again(t, mine, p.cache, table, kb, vb, k, min(k + KT, k1), lim[t], c, lane);
            }
        }
        /* the waves' results of a tile at a time; each wave adds up and stores some of the dimensions */
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            __syncthreads();
            l_char* mine = lds + wave * W::SUMS;
#pragma unroll
            for (int i = 0; i < W::DT; ++i) *(l_f4*)(mine + (i * WAVE + lane) * 16) = w.o[t][i];
            *(l_float*)(mine + (W::DT * WAVE + lane) * 16) = w.m[t];
            *(l_float*)(mine + (W::DT * WAVE + lane) * 16 + 4) = w.l[t];
            __syncthreads();
            float m = NEG_INF, l = 0.f, f[AW];
#pragma unroll
            for (int x = 0; x < AW; ++x) m = fmaxf(m, *(const l_float*)(lds + x * W::SUMS + (W::DT * WAVE + lane) * 16));
            const float base = m == NEG_INF ? 0.f : m * c;
#pragma unroll
            for (int x = 0; x < AW; ++x) {
                const l_float* ml = (const l_float*)(lds + x * W::SUMS + (W::DT * WAVE + lane) * 16);
                f[x] = __builtin_amdgcn_exp2f(ml[0] * c - base);
                l = fmaf(ml[1], f[x], l);
            }
            const int row = row0 + 16 * t + col, tok = s.t0 + row / G, qh = head * G + row % G;
            const float inv = inverse_of(l);
#pragma unroll
            for (int i0 = 0; i0 < W::DT; i0 += AW) {
                const int i = i0 + wave;
                f4_t sum = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < AW; ++x) {
                    const f4_t v = *(const l_f4*)(lds + x * W::SUMS + (i * WAVE + lane) * 16);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[j] = fmaf(v[j], f[x], sum[j]);
                }
                if (row > last) continue;
                if (whole) {
                    char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
                    *(u32x2*)(out + (16 * i + 4 * g) * 2) =
                        u32x2{pack2<FMT>(sum[0] * inv, sum[1] * inv), pack2<FMT>(sum[2] * inv, sum[3] * inv)};
                } else {
                    float* to = pl.part + ((int64_t)(2 * share + (o == 0)) * R + row - row0) * (D + 4);
                    *(f4_t*)(to + 16 * i + 4 * g) = sum;
                }
            }
            if (wave == 0 && g == 0 && row <= last) {
                if (whole) {
                    if (p.lse) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(m, l, p.scale);
                } else {
                    float* to = pl.part + ((int64_t)(2 * share + (o == 0)) * R + row - row0) * (D + 4);
                    to[D] = m, to[D + 1] = l;
                }
            }
        }
        __syncthreads();                                        /* the waves' values may go where their results were */
        left -= take;
        if (left <= 0) return;
        o = 0;
        if (++tile < s.tiles) continue;
        tile = 0;
        if (++head < N) continue;
        head = 0;
        do {
            if (++b >= p.n_seqs) return;
            s = seq_at(p, R, b);
        } while (!s.tiles);
    }
}

/* Rows whose tile lies in several shares: the shares' parts in order, a wave per (token, head). */
template <int FMT, int D>
__global__ __launch_bounds__(AT) void k_paged_join(wsr_paged p, PagedPlan pl, int64_t first) {
    constexpr int E = D / WAVE;
    const int64_t at = first + (int64_t)blockIdx.x * AW + wsr::wave_in_block();
    const int lane = threadIdx.x % WAVE;
    if (at >= (int64_t)p.n_tokens * p.n_heads) return;
    const int tok = (int)(at / p.n_heads), qh = (int)(at % p.n_heads), G = p.n_heads / p.n_kv_heads, R = pl.rows;
    const int b = seq_of(p.starts, p.n_seqs, tok).seq;
    if (b < 0) return;
    const Line line = line_of(p, pl, lane);
    int64_t x = 0;
    for (int b0 = 0; b0 <= b; b0 += WAVE) {
        const int64_t to = costs_to(p, R, b0, x, lane);
        if (b >= b0 + WAVE) x = lane64(to, WAVE - 1);
        else if (b > b0) x = lane64(to, b - b0 - 1);
    }
    const Seq s = seq_at(p, R, b);
    const int row = (tok - s.t0) * G + qh % G, tile = row / R;
    if (tok < s.t0 || tok >= s.t0 + s.n) return;
    x += qh / G * s.cost + before_tile(s, R, tile);
    const int w0 = line.share_of(x), w1 = line.share_of(x + tile_cost(s, R, tile) - 1);
    if (w0 == w1) return;
    const float c = p.scale * LOG2E;
    float m = NEG_INF, l = 0.f, o[E] = {};
    for (int w = w0; w <= w1; ++w) {
        const float* from = pl.part + ((int64_t)(2 * w + (w == w0)) * R + row - tile * R) * (D + 4);
        const float pm = from[D], ps = from[D + 1], top = fmaxf(m, pm), base = top == NEG_INF ? 0.f : top * c;
        const float a = __builtin_amdgcn_exp2f(m * c - base), f = __builtin_amdgcn_exp2f(pm * c - base);
        l = l * a + ps * f;
        m = top;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * a + from[E * lane + e] * f;
    }
    const float inv = inverse_of(l);
    char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
    if constexpr (E == 4) ((u32x2*)out)[lane] = u32x2{pack2<FMT>(o[0] * inv, o[1] * inv), pack2<FMT>(o[2] * inv, o[3] * inv)};
    else if constexpr (E == 2) ((uint32_t*)out)[lane] = pack2<FMT>(o[0] * inv, o[1] * inv);
    else ((uint16_t*)out)[lane] = (uint16_t)pack2<FMT>(o[0] * inv, 0.f);
    if (p.lse && lane == 0) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(m, l, p.scale);
}

/* ---- host ------------------------------------------------------------------------------------------ */

static PagedPlan paged_plan(const wsr_paged& p) {
    PagedPlan pl{};
    pl.rows = 16;
    pl.shares = 512;
    /* n / d = (n * M) >> (31 + s), 2^s >= d, M = 2^(31 + s) / d + 1, for n < 2^31: M d is over 2^(31 + s) by at most d */
    int s = 0;
    while ((int64_t)1 << s < p.cache.page_size) ++s;
    pl.magic = ((uint64_t)1 << (31 + s)) / p.cache.page_size + 1;
    pl.shift = 31 + s;
    return pl;
}

size_t paged_workspace(const wsr_paged& p) {
    const PagedPlan pl = paged_plan(p);
    return (size_t)2 * pl.shares * pl.rows * (p.head_dim + 4) * sizeof(float);
}

template <int FMT, int D>
static hipError_t launch_dim(const wsr_paged& p, const PagedPlan& pl, hipStream_t s) {
    hipLaunchKernelGGL((k_paged<FMT, D, 1>), dim3((unsigned)pl.shares), dim3(AT), 0, s, p, pl);
    hipError_t e = hipGetLastError();
    const int64_t rows = (int64_t)p.n_tokens * p.n_heads;
    for (int64_t first = 0; e == hipSuccess && first < rows; first += most_blocks(AT) * AW) {
        const int64_t n = std::min((rows - first + AW - 1) / AW, most_blocks(AT));
        hipLaunchKernelGGL((k_paged_join<FMT, D>), dim3((unsigned)n), dim3(AT), 0, s, p, pl, first);
        e = hipGetLastError();
    }
    return e;
}

template <int FMT>
static hipError_t launch_fmt(const wsr_paged& p, const PagedPlan& pl, hipStream_t s) {
    return p.head_dim == 64 ? launch_dim<FMT, 64>(p, pl, s) : p.head_dim == 128 ? launch_dim<FMT, 128>(p, pl, s) : launch_dim<FMT, 256>(p, pl, s);
}

hipError_t launch_paged(const wsr_paged& p, void* ws, hipStream_t s) {
    PagedPlan pl = paged_plan(p);
    pl.part = static_cast<float*>(ws);
    return p.fmt == WSR_F16 ? launch_fmt<WSR_F16>(p, pl, s) : launch_fmt<WSR_BF16>(p, pl, s);
}

}  // namespace wsr_serve
