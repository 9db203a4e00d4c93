/*
 * wsr_paged.hip - attention of each sequence's newest tokens over its pages.
 *
 * A query row is one (token, query head); the rows of a sequence and key head, tokens times G = n_heads / n_kv_heads, go in
 * tiles of R.  A unit of work is a tile of one key head; units that are long against what all of them come to are cut along
 * the keys into equal parts, by the lengths that the device holds, so that any mix of lengths fills the chip.  A unit in one
 * part is stored at once; of the others each part leaves a maximum, a sum and an unnormalised fp32 row, which k_paged_join
 * adds up.  Where the host sees that no sequence can be long enough to be cut, there is one launch.
 *
 * A wave walks blocks of 32 keys with a running maximum and sum:
 *
 *   S^T = K Q^T   (v_mfma 16x16x32: 16 keys x 16 rows, each lane one row and four keys)
 *   P   = exp2((S - max) scale log2 e),  O^T += V^T P^T with P still in the registers of S: the lane layout of S^T is
 *         the operand layout of P^T when V's keys are taken in the same order.  P is rounded to the values' 16 bits, as the
 *         instruction takes both operands in one type, and its sum is not: in f16 0.00025 to 0.00027 from 64 bits where
 *         outputs alone are 0.00021, in bf16 0.0019 to 0.0022 and 0.0017.  (A second operand with P's rest would leave the
 *         latter for twice these products.)
 *
 * Keys and values are loaded as whole rows, a wave's 64 lanes of 16 bytes side by side, into registers, which hold more on
 * their way than LDS could, and turned into operands by the wave's own 32 rows of LDS: first the keys, then, by transposing
 * reads, the values.  (Loaded straight in operand layout, 64 bytes of 16 keys at a time, 7 sequences of up to 65536 keys took
 * 295 us, so 259; and whole rows gain from the hint that they are read once, 292 without it, which the others lose by.)  No wave
 * waits for another before the end, where those of a workgroup, who take blocks in turn, add up.
 *
 * Bound by HBM: those 7, 1577 MB of keys, 248 us (6.4 TB/s), 32 of up to 4096 62 (320 MB, 5.1 TB/s).  Short ones are
 * latency, lengths, pages, keys and the join in turn: one of 500 keys 8.1 us, one of 2000 12, 32771 31 (134 MB).
 * Tiles of 64 and 128 rows: wsr_paged_rows.hip.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_paged.h"

namespace wsr_serve {

constexpr int KT = 32;                        /* keys of a wave's block */
typedef short s4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char l_char;
typedef __attribute__((address_space(3))) s4_t l_s4;
typedef __attribute__((address_space(3))) f4_t l_f4;
typedef __attribute__((address_space(3))) float l_float;
typedef __attribute__((address_space(3))) u32x4 l_u32x4;

/* The running maximum is only moved when a row's scores pass it by 2^LAZY: until then its probabilities are taken
   against the old one (at most 2^LAZY, exact after the division by their sum). */
constexpr float LAZY = 8.f;

/* ---- a wave's walk ----------------------------------------------------------------------------------- */

template <int FMT, int D, int RT, bool ONCE>  /* RT: tiles of 16 rows; ONCE: hinted that keys are read once */
struct Walk {
    static constexpr int KS = D / 32, DT = D / 16, R = 16 * RT;
    static constexpr int PIECES = D / 8, ROW = 2 * D;           /* 16-byte pieces of a key, and its bytes */
    static constexpr int AT_ONCE = WAVE / PIECES, LOADS = KT / AT_ONCE;   /* keys of a load, loads of a block */
    static constexpr int BUFFER = KT * ROW;                     /* bytes of a wave's block in LDS */
    static constexpr int SUMS = WAVE * (DT + 1) * 16;           /* bytes of a wave's results in LDS, of 16 rows */
    static constexpr int ROOM = BUFFER > SUMS ? BUFFER : SUMS;

    u32x4 q[RT][KS];
    f4_t o[RT][DT];
    float m[RT], l[RT];
    u32x4 k[LOADS], v[LOADS];                                   /* key AT_ONCE i + l / PIECES, piece l % PIECES */
    int64_t off;                                                /* of the block's key l % 32 */
    int entry, slot;                                            /* and of the next one's */
    uint32_t there;                                             /* the block's keys that are on a page */

    /* Piece x of key y lies at x ^ swz(y) of its row: the 16 keys of a read of keys, and the eight keys times two pieces of half
       a transposing read, lie on the 64 banks once each. */
    static __device__ __forceinline__ int kswz(int key) { return D == 64 ? key >> 1 & 7 : key & 15; }
    static __device__ __forceinline__ int vswz(int key) {
        return D == 64 ? (key >> 1 & 1) << 1 | (key >> 2 & 1) << 2 : (key & 3) << 2 | (key >> 2 & 1) << 1;
    }

    __device__ __forceinline__ void look_up(const wsr_pages& c, const PagedPlan& pl, const int32_t* table, int at, int k1, int lane) {
        const int key = min(at + lane % 32, k1 - 1);
        const int page = (int)((uint64_t)key * pl.magic >> pl.shift);
        slot = key - page * c.page_size;
        entry = table[page];
    }
    /* Where the block's keys are; those that are not there repeat the first that is, or, where none is, `some` readable row. */
    __device__ __forceinline__ void place(const wsr_pages& c, int at, int k1, int lane) {
        there = (uint32_t)__ballot((uint32_t)entry < (uint32_t)c.n_pages && at + lane % 32 < k1);
        off = entry * c.page_stride + slot * c.tok_stride;
        if (!there) {
            off = 0;
        } else if (there != 0xffffffffu) {
            const int f = __builtin_ctz(there);
            const int64_t first = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(off >> 32), f) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)off, f));
            if (!(there >> lane % 32 & 1)) off = first;
        }
    }
    __device__ __forceinline__ void load(u32x4 (&to)[LOADS], const char* base, const char* some, int lane) const {
        const char* from = (there ? base : some) + lane % PIECES * 16;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
        {
            const u32x4* at = (const u32x4*)(from + __shfl((long long)off, AT_ONCE * i + lane / PIECES));
            if constexpr (ONCE) to[i] = __builtin_nontemporal_load(at);
            else to[i] = *at;
        }
    }
    /* The block's rows are turned in LDS: keep_keys(), scores(), keep_values(), weigh(), each after a wave_fence(). */
    __device__ __forceinline__ void keep_keys(l_char* buf, int lane) const {
        wave_fence();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key = AT_ONCE * i + lane / PIECES;
            *(l_u32x4*)(buf + key * ROW + (lane % PIECES ^ kswz(key)) * 16) = k[i];
        }
    }
    __device__ __forceinline__ void keep_values(l_char* buf, int lane) const {
        wave_fence();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key = AT_ONCE * i + lane / PIECES;
            *(l_u32x4*)(buf + key * ROW + (lane % PIECES ^ vswz(key)) * 16) = v[i];
        }
    }

    __device__ __forceinline__ void scores(f4_t (&s)[RT][2], const l_char* buf, int lane) const {
        wave_fence();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int t = 0; t < RT; ++t) s[t][h] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const int key = lane % 16;
                const u32x4 f = *(const l_u32x4*)(buf + (16 * h + key) * ROW + ((4 * i + lane / 16) ^ kswz(key)) * 16);
#pragma unroll
                for (int t = 0; t < RT; ++t) s[t][h] = wsr_step::mma16<FMT>(f, q[t][i], s[t][h]);
            }
        }
    }
    /* The scores' block, keys at .. + 31: those in `seen` are there, and this lane's row sees those before lim. */
    __device__ __forceinline__ void weigh(f4_t (&s)[RT][2], uint32_t seen, bool masked, const int (&lim)[RT], int at, float c,
                                          const l_char* buf, int lane) {
        const int g = lane / 16;
        u32x4 pt[RT];
        wave_fence();
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
        /* the lane's part of a transposing read: keys 4 g .. + 3, 16 dimensions */
        const int key = 4 * g + lane % 16 / 4;
        const l_char* from = buf + key * ROW + lane % 2 * 8;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            u32x4 f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                              (l_s4*)(from + 16 * h * ROW + ((2 * i + lane % 4 / 2) ^ vswz(key)) * 16)));
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

/* Waves per SIMD that the registers of a form allow. */
constexpr int waves_of(int D, int RT) { return D == 256 ? 1 : RT == 2 ? D == 64 ? 3 : 2 : D == 64 ? 4 : 3; }

template <int FMT, int D, int RT, int NW, bool ONCE>     /* NW: waves */
__global__ __launch_bounds__(NW * WAVE) __attribute__((amdgpu_waves_per_eu(waves_of(D, RT)))) void k_paged(wsr_paged p, PagedPlan pl) {
    typedef Walk<FMT, D, RT, ONCE> W;
    constexpr int R = W::R, STEP = KT * NW;
    __shared__ u32x4 lds_room[NW * W::ROOM / 16];
    l_char* lds = (l_char*)lds_room;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    const int G = p.n_heads / p.n_kv_heads, N = p.n_kv_heads;
    const float c = p.scale * LOG2E;
    Place at_place;
    if (!find(p, pl, blockIdx.x, false, at_place)) return;
    const int b = at_place.seq, parts = at_place.parts, part = at_place.at % parts, unit = at_place.at / parts;
    const int head = unit % N, tile = unit / N;
    const Seq s = at_place.s;
    const int row0 = tile * R, last = min(row0 + R, s.rows) - 1, past = s.len - s.n;
    const int seen = max(past + last / G + 1, 0);
    /* equal parts of whole rounds of blocks */
    const int each = ((seen + parts - 1) / parts + STEP - 1) / STEP * STEP;
    const int k0 = (int)min((int64_t)part * each, (int64_t)seen), k1 = seen - k0 > each ? k0 + each : seen;
    const char* kb = (const char*)p.cache.k + head * p.cache.head_stride;
    const char* vb = (const char*)p.cache.v + head * p.cache.head_stride;
    const int32_t* table = (const int32_t*)((const char*)p.cache.table + b * p.cache.table_stride);
    W w;
    l_char* buf = lds + wave * W::ROOM;
    int at = k0 + wave * KT;
    if (at < k1) w.look_up(p.cache, pl, table, at, k1, lane);
    int lim[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int row = min(row0 + 16 * t + col, last), tok = row / G;
        lim[t] = past + tok + 1;
        const char* qr = (const char*)p.q + (s.t0 + tok) * p.q_tok_stride + (head * G + row - tok * G) * p.q_head_stride;
#pragma unroll
        for (int i = 0; i < W::KS; ++i) w.q[t][i] = ((const u32x4*)qr)[4 * i + g];
#pragma unroll
        for (int i = 0; i < W::DT; ++i) w.o[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
        w.m[t] = NEG_INF, w.l[t] = 0.f;
    }
    const int all = past + row0 / G + 1;                        /* keys that every row sees */
    const char* some = (const char*)p.q + s.t0 * p.q_tok_stride + head * G * p.q_head_stride;
    if (at < k1) {
        w.place(p.cache, at, k1, lane);
        w.load(w.k, kb, some, lane);
        w.load(w.v, vb, some, lane);
        w.look_up(p.cache, pl, table, at + STEP, k1, lane);
        uint32_t there = w.there;
        f4_t sc[RT][2];
        /* the next block's keys (values) are on their way as soon as one's are in LDS */
#pragma unroll 1
        for (; at + STEP < k1; at += STEP) {
            w.keep_keys(buf, opaque(lane));
            w.place(p.cache, at + STEP, k1, lane);
            w.load(w.k, kb, some, opaque(lane));
            w.scores(sc, buf, opaque(lane));
            w.keep_values(buf, opaque(lane));
            w.load(w.v, vb, some, opaque(lane));
            w.look_up(p.cache, pl, table, at + 2 * STEP, k1, lane);
            w.weigh(sc, there, there != 0xffffffffu || at + KT > all, lim, at, c, buf, opaque(lane));
            there = w.there;
        }
        w.keep_keys(buf, lane);
        w.scores(sc, buf, lane);
        w.keep_values(buf, lane);
        w.weigh(sc, there, there != 0xffffffffu || at + KT > all, lim, at, c, buf, lane);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        w.l[t] = wsr::xchg_add<1>(wsr::xchg_add<0>(w.l[t]));
        const bool mine = w.broken(t) && w.l[t] == w.l[t];      /* a NaN sum makes all of the row NaN as it is */
        if (__ballot(mine)) {
            if (mine)
#pragma unroll
                for (int i = 0; i < W::DT; ++i) w.o[t][i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int k = k0 + wave * KT; k < k1; k += STEP)
                w.again(t, mine, p.cache, table, kb, vb, k, min(k + KT, k1), lim[t], c, lane);
        }
    }
    /* the waves' results of 16 rows at a time; each wave adds up and stores some of the dimensions */
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t) __syncthreads();
        else wave_fence();
        l_char* mine = lds + wave * W::ROOM;
#pragma unroll
        for (int i = 0; i < W::DT; ++i) *(l_f4*)(mine + (i * WAVE + lane) * 16) = w.o[t][i];
        *(l_float*)(mine + (W::DT * WAVE + lane) * 16) = w.m[t];
        *(l_float*)(mine + (W::DT * WAVE + lane) * 16 + 4) = w.l[t];
        __syncthreads();
        const int row = row0 + 16 * t + col, tok = s.t0 + row / G, qh = head * G + row % G;
        if (wave >= W::DT) continue;
        float m = NEG_INF, l = 0.f;
#pragma unroll
        for (int x = 0; x < NW; ++x) m = fmaxf(m, *(const l_float*)(lds + x * W::ROOM + (W::DT * WAVE + lane) * 16));
        const float base = m == NEG_INF ? 0.f : m * c;
        constexpr int PER = (W::DT + NW - 1) / NW;
        f4_t sum[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) sum[i] = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            const l_char* from = lds + x * W::ROOM;
            const l_float* ml = (const l_float*)(from + (W::DT * WAVE + lane) * 16);
            const float f = __builtin_amdgcn_exp2f(ml[0] * c - base);
            l = fmaf(ml[1], f, l);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const f4_t v = *(const l_f4*)(from + ((wave + NW * i) * WAVE + lane) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[i][j] = fmaf(v[j], f, sum[i][j]);
            }
        }
        if (row > last) continue;
        if (parts == 1) {
            const float inv = inverse_of(l);
            char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                *(u32x2*)(out + (16 * (wave + NW * i) + 4 * g) * 2) =
                    u32x2{pack2<FMT>(sum[i][0] * inv, sum[i][1] * inv), pack2<FMT>(sum[i][2] * inv, sum[i][3] * inv)};
            if (p.lse && wave == 0 && g == 0) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(m, l, p.scale);
        } else {
            const int slot = at_place.slot + at_place.at;
            if ((uint32_t)slot >= (uint32_t)pl.slots) continue;
            float* to = pl.part + ((int64_t)slot * R + row - row0) * (D + 4);
#pragma unroll
            for (int i = 0; i < PER; ++i) *(f4_t*)(to + 16 * (wave + NW * i) + 4 * g) = sum[i];
            if (wave == 0 && g == 0) to[D] = m, to[D + 1] = l;
        }
    }
}

/* The cut, and the items and slots before each sequence, by one workgroup, a lane to each of 1024 sequences at a time.  Starts
   that fall may count more items than 32 bits hold; sums then stay at LINE_END. */
constexpr int NT = 1024, NW = NT / WAVE;
__global__ __launch_bounds__(NT) void k_paged_line(wsr_paged p, PagedPlan pl) {
    __shared__ float keys[NW], units[NW];
    __shared__ int64_t all[2][NW], cuts[2][NW];                 /* of the waves, of one pass of the loop and the next */
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), N = p.n_kv_heads;
    Cut cut{1.f, 0.f};
    if (!pl.whole) {
        Sums sums{0.f, 0.f};
#pragma unroll 4
        for (int b = threadIdx.x; b < p.n_seqs; b += NT) sums.add(seq_at(p, pl.rows, b), N);
        sums.keys = wsr::wave_sum(sums.keys), sums.units = wsr::wave_sum(sums.units);
        if (lane == 0) keys[wave] = sums.keys, units[wave] = sums.units;
        __syncthreads();
        sums = Sums{0.f, 0.f};
        for (int w = 0; w < NW; ++w) sums.keys += keys[w], sums.units += units[w];
        cut = cut_of(pl, sums);
        if (threadIdx.x == 0) pl.line->cut = cut;
    }
    int64_t items = 0, slots = 0;
    Seq next = seq_at(p, pl.rows, min((int)threadIdx.x, p.n_seqs - 1));
    for (int b0 = 0, odd = 0; b0 < p.n_seqs; b0 += NT, odd ^= 1) {
        const Seq s = next;
        const int b = b0 + threadIdx.x;
        if (b0 + NT < p.n_seqs) next = seq_at(p, pl.rows, min(b + NT, p.n_seqs - 1));
        const int parts = pl.whole ? 1 : parts_of(s, cut);
        const int mine = b < p.n_seqs ? (int)min((int64_t)(s.tiles * N) * parts, (int64_t)LINE_END / WAVE) : 0, cutting = parts > 1 ? mine : 0;
        const int to = scan32(mine), cuts_to = scan32(cutting);
        if (lane == WAVE - 1) all[odd][wave] = to, cuts[odd][wave] = cuts_to;
        __syncthreads();
        int64_t i = items + to - mine, c = slots + cuts_to - cutting;
        for (int w = 0; w < NW; ++w) {
            if (w < wave) i += all[odd][w], c += cuts[odd][w];
            items += all[odd][w], slots += cuts[odd][w];
        }
        if (b < p.n_seqs) pl.line->upto[b] = Upto{(int32_t)min(i, (int64_t)LINE_END), (int32_t)min(c, (int64_t)LINE_END)};
    }
}

/* Rows whose unit is cut.  A part's row takes D / 4 lanes: where rows are many, W = 1, a wave has a row in each of its groups of
   so many lanes (2 chunks of up to 512 tokens 11 us, with one row a wave 16); where they are few, four waves take the parts
   of one row, a group each.  AHEAD parts are loaded at a time. */
constexpr int JT = 256, JW = JT / WAVE;
template <int FMT, int D, int W>
__global__ __launch_bounds__(JT) __attribute__((amdgpu_waves_per_eu(W == 1 ? 8 : 4))) void k_paged_join(wsr_paged p, PagedPlan pl) {
    constexpr int LANES = D / 4, SIDE = WAVE / LANES, AHEAD = 4, ROWS = W == 1 ? SIDE : 1, APART = W == 1 ? 1 : SIDE * W;
    __shared__ f4_t sums[JW][LANES];
    __shared__ float stats[JW][2];
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), turn = wave % W, group = lane / LANES, x = lane % LANES;
    const int64_t first = ((int64_t)blockIdx.x * (JW / W) + wave / W) * ROWS, rows = (int64_t)p.n_tokens * p.n_heads;
    if (first >= rows) return;                                  /* of W = 4, all of the workgroup */
    const int64_t at = min(first + (W == 1 ? group : 0), rows - 1);
    const int tok = (int)(at / p.n_heads), qh = (int)(at % p.n_heads), G = p.n_heads / p.n_kv_heads, R = pl.rows;
    int parts = 1;
    const float* from = pl.part;
    const int64_t step = (int64_t)R * (D + 4);
    const int last = (int)(min(first + ROWS - 1, rows - 1) / p.n_heads);
    for (int t = (int)(first / p.n_heads); t <= last; ++t) {    /* the wave's tokens, most often one */
        const int b = seq_of(p.starts, p.n_seqs, t).seq;
        Place o_place;
        if (b < 0 || !find(p, pl, b, true, o_place) || o_place.parts == 1 || t != tok) continue;
        const int row = (tok - o_place.s.t0) * G + qh % G, slot = o_place.slot + (row / R * p.n_kv_heads + qh / G) * o_place.parts;
        if (slot < 0 || slot > pl.slots - o_place.parts) continue;
        parts = o_place.parts;
        from = pl.part + ((int64_t)slot * R + row % R) * (D + 4);
    }
    if (__ballot(parts > 1) == 0) return;
    if (parts == 1) parts = 0;
    const float c = p.scale * LOG2E;
    float m = NEG_INF, l = 0.f;
    f4_t o = f4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i = W == 1 ? 0 : turn * SIDE + group; i < parts; i += AHEAD * APART) {
        float pm[AHEAD], ps[AHEAD];
        f4_t po[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int j = i + k * APART;
            const float* w = from + min(j, parts - 1) * step;
            pm[k] = j < parts ? w[D] : NEG_INF, ps[k] = j < parts ? w[D + 1] : 0.f;
            po[k] = j < parts ? *(const f4_t*)(w + 4 * x) : f4_t{0.f, 0.f, 0.f, 0.f};
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) top = fmaxf(top, pm[k]);
        const float base = top == NEG_INF ? 0.f : top * c, a = __builtin_amdgcn_exp2f(m * c - base);
        l *= a;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= a;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float f = __builtin_amdgcn_exp2f(pm[k] * c - base);
            l = fmaf(ps[k], f, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(po[k][e], f, o[e]);
        }
        m = top;
    }
    if constexpr (W > 1) {
        auto add = [&](float m2, float l2, f4_t o2) {
            const float top = fmaxf(m, m2), base = top == NEG_INF ? 0.f : top * c;
            const float a = __builtin_amdgcn_exp2f(m * c - base), f = __builtin_amdgcn_exp2f(m2 * c - base);
            l = l * a + l2 * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = o[e] * a + o2[e] * f;
            m = top;
        };
#pragma unroll
        for (int d = LANES; d < WAVE; d *= 2) {
            f4_t o2;
#pragma unroll
            for (int e = 0; e < 4; ++e) o2[e] = __shfl_xor(o[e], d);
            add(__shfl_xor(m, d), __shfl_xor(l, d), o2);
        }
        if (lane < LANES) sums[wave][x] = o;
        if (lane == 0) stats[wave][0] = m, stats[wave][1] = l;
        __syncthreads();
        if (turn || lane >= LANES) return;
#pragma unroll
        for (int w = 1; w < W; ++w) add(stats[w][0], stats[w][1], sums[w][x]);
    }
    if (parts == 0 || first + (W == 1 ? group : 0) >= rows) return;
    const float inv = inverse_of(l);
    char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
    ((u32x2*)out)[x] = u32x2{pack2<FMT>(o[0] * inv, o[1] * inv), pack2<FMT>(o[2] * inv, o[3] * inv)};
    if (p.lse && x == 0) p.lse[at] = lse_of(m, l, p.scale);
}

/* ---- host ------------------------------------------------------------------------------------------ */

/* Sequences times key heads below which units are few: one launch then pays up to 768 keys (one sequence of 500 11.7 us in
   two, 8.1 in one with twelve waves a unit; of 1000 11.5 and 11.8), and beyond it up to 1536 (63 of 1000 33.4 us in two, 31 in
   one; 64 of 500 25.8 and 18.5, with twelve waves a unit 19.7). */
constexpr int FEW_UNITS = 256, WHOLE = 768;
/* Rows up to which a row's parts are joined by four waves: 32 rows of 86 parts 15 us by one wave each, so 6. */
constexpr int FEW_ROWS = 2048;

/* Sequences up to which every wave finds its work by itself: past 192 k_paged_line pays (heads of 128, 32 on 8, up to 300 keys
   of 2000: 192 sequences 43.4 us without it and 39.2, 1024 341 and 144, 4096 4264 and 569; 8 heads on 1 21.1 and 20.5, 85 and 31), in
   a call that is otherwise one launch past 512 (up to 300 keys: 512 sequences 80.6 and 69.5, 8 heads on 1 16.4 and 17.8, 1024 187
   and 133, 31.1 and 26.5). */
constexpr int MANY = 192, MANY_WHOLE = 512;
/* Bytes of the workspace that k_paged_line writes, before the parts; whole or not, as a call of fewer tokens may not be. */
static size_t line_bytes(const wsr_paged& p) {
    return p.n_seqs <= MANY ? 0 : (sizeof(Cut) + sizeof(Upto) * p.n_seqs + 255) / 256 * 256;
}

/* Rows of a tile, one height for the whole call, as the host does not know which sequence has how many: as many as a sequence's
   fill, on average; 128 where there are tiles enough of them (a chunk of 512 tokens of
   32 heads on 8, 128 tiles, 18.6 us with 128 rows and 15.5 with 64; two of up to 512 behind 4096, 216 tiles, 72 and 81), of
   heads of 256, whose workgroups are one to a CU, half as many (16 on 4: 4 chunks of up to 64, 32 tiles, 43 and 30; two of up to
   512 behind 4096, 108 tiles, 87 and 112, with 32 rows 173). */
static int tile_rows(const wsr_paged& p) {
    const int64_t rows = (int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads), n = p.n_seqs;
    if (rows <= 16 * n) return 16;
    if (rows <= 32 * n) return 32;
    return rows <= 64 * n || p.n_kv_heads * (rows / 128) < (p.head_dim == 256 ? 80 : 160) ? 64 : 128;
}

/* Units of a call, at most. */
static int64_t most_units(const wsr_paged& p, const PagedPlan& pl) {
    const int64_t rows = (int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads);
    return p.n_kv_heads * (rows / pl.rows + std::min(p.n_seqs, p.n_tokens));
}

static int32_t held_of(int32_t rows, int32_t head_dim) { return 256 * (rows <= 32 ? waves_of(head_dim, rows / 16) : head_dim == 256 ? 1 : 2); }
constexpr int SPARE = 64;                     /* slots, for what fp32 sums of lengths may be off by */
static PagedPlan paged_plan(const wsr_paged& p) {
    PagedPlan pl{};
    pl.rows = tile_rows(p);
    pl.held = held_of(pl.rows, p.head_dim);
    /* parts come to what the chip holds where units are few, to twice that elsewhere */
    pl.slots = (most_units(p, pl) <= few_units(pl) ? 1 : 2) * pl.held + SPARE;
    pl.whole = p.max_len <= ((int64_t)p.n_kv_heads * std::min(p.n_seqs, p.n_tokens) < FEW_UNITS ? WHOLE : 2 * WHOLE);
    /* n / d = (n * M) >> (31 + s), 2^s >= d, M = 2^(31 + s) / d + 1, for n < 2^31: M d is over 2^(31 + s) by at most d */
    int s = 0;
    while ((int64_t)1 << s < p.cache.page_size) ++s;
    pl.magic = ((uint64_t)1 << (31 + s)) / p.cache.page_size + 1;
    pl.shift = 31 + s;
    return pl;
}

/* What the call needs, and any of fewer tokens, whose tiles may be smaller and more. */
size_t paged_workspace(const wsr_paged& p) {
    const PagedPlan pl = paged_plan(p);
    if (p.max_len <= WHOLE) return std::max<size_t>(256, line_bytes(p));
    size_t rows = (size_t)pl.slots * pl.rows;
    for (int32_t r = 16; r < pl.rows; r *= 2) rows = std::max(rows, (size_t)(2 * held_of(r, p.head_dim) + SPARE) * r);
    return line_bytes(p) + rows * (p.head_dim + 4) * sizeof(float);
}

/* Workgroups of the first launch. */
static int64_t paged_blocks(const wsr_paged& p, const PagedPlan& pl) { return most_units(p, pl) + (pl.whole ? 0 : pl.slots); }
bool paged_fits(const wsr_paged& p) { return paged_blocks(p, paged_plan(p)) <= most_blocks(4 * WAVE); }

template <int FMT, int D>
static hipError_t launch_dim(const wsr_paged& p, const PagedPlan& pl, hipStream_t s) {
    const int64_t blocks = paged_blocks(p, pl);
    const dim3 grid((unsigned)blocks), threads(4 * WAVE);
    /* whether a sequence's rows are one tile, on average: the hint that its keys are read once, right for most of them then.  Of
       others it costs time alone (63 tokens and a chunk of 200 of 32 heads on 8 154 us, in two calls 149). */
    const bool once = (int64_t)p.n_tokens * (p.n_heads / p.n_kv_heads) <= (int64_t)pl.rows * p.n_seqs;
    hipError_t e;
    if (pl.line) {
        hipLaunchKernelGGL(k_paged_line, dim3(1), dim3(NT), 0, s, p, pl);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (pl.rows > 32) {
        e = launch_paged_rows(p, pl, pl.rows / 32, once, blocks, s);
    } else {
        if (pl.rows == 16 && pl.whole && D < 256 && (int64_t)p.n_kv_heads * p.n_seqs < FEW_UNITS)
            hipLaunchKernelGGL((k_paged<FMT, D, 1, (D < 256 ? 12 : 4), true>), grid, dim3(12 * WAVE), 0, s, p, pl);
        else if (pl.rows == 16) hipLaunchKernelGGL((k_paged<FMT, D, 1, 4, true>), grid, threads, 0, s, p, pl);
        else if (once) hipLaunchKernelGGL((k_paged<FMT, D, 2, 4, true>), grid, threads, 0, s, p, pl);
        else hipLaunchKernelGGL((k_paged<FMT, D, 2, 4, false>), grid, threads, 0, s, p, pl);
        e = hipGetLastError();
    }
    if (e != hipSuccess || pl.whole) return e;
    const int64_t rows = (int64_t)p.n_tokens * p.n_heads;       /* at most 2^25: one launch */
    if (rows <= FEW_ROWS) hipLaunchKernelGGL((k_paged_join<FMT, D, JW>), dim3((unsigned)rows), dim3(JT), 0, s, p, pl);
    else hipLaunchKernelGGL((k_paged_join<FMT, D, 1>), dim3((unsigned)((rows + JT * 4 / D - 1) / (JT * 4 / D))), dim3(JT), 0, s, p, pl);
    return hipGetLastError();
}

template <int FMT>
static hipError_t launch_fmt(const wsr_paged& p, const PagedPlan& pl, hipStream_t s) {
    return p.head_dim == 64 ? launch_dim<FMT, 64>(p, pl, s) : p.head_dim == 128 ? launch_dim<FMT, 128>(p, pl, s) : launch_dim<FMT, 256>(p, pl, s);
}

hipError_t launch_paged(const wsr_paged& p, void* ws, hipStream_t s) {
    PagedPlan pl = paged_plan(p);
    char* at = static_cast<char*>(ws);
    pl.part = reinterpret_cast<float*>(at + line_bytes(p));
    if (p.n_seqs > (pl.whole ? MANY_WHOLE : MANY)) pl.line = reinterpret_cast<Line*>(at);
    return p.fmt == WSR_F16 ? launch_fmt<WSR_F16>(p, pl, s) : launch_fmt<WSR_BF16>(p, pl, s);
}

}  // namespace wsr_serve
