/*
 * wsr_logprobs.hip - log probabilities of given tokens, with rank, entropy and the most likely alternatives.
 *
 *   p = softmax(l / T):  log p_x = (l_x - m) / T - log s,  s = sum exp((l - m) / T),
 *   entropy = log s + sum p (m - l) / T
 *
 * One read of a row: every lane keeps a maximum of its own and the two sums against it, and the wave how many logits come
 * before the given token's.  A row is a workgroup's, or, where rows are few, several parts' that a second launch joins.
 * (Equal shares of all rows' chunks, which begin and end inside rows, cost a second set of alternatives in every workgroup:
 * 4001 rows of 25001 with five 103 us, so 85, and 2055 of 50257 with one 80 and 76.)
 *
 * The n largest: a wave keeps its best 64 in order, one per lane, as 64-bit keys (the logit's bits in an order of whole
 * numbers, then the index from the top, so that equal logits go by index).  Logits that pass the n-th key, which after
 * the first few hundred are rare, are collected in LDS and merged in 64 at a time, sorted by compare-and-swap networks
 * over the wave.  The first chunks' threshold is the n-th largest of the lanes' maxima, which n logits reach.  A single
 * alternative is a lane's largest and needs none of this.
 *
 * Bound by HBM where rows are many: 2055 rows of 50257, 413 MB, 70 to 72 us without alternatives (5.8 TB/s; eleven
 * instructions a logit), 75 with one, 82 with five, where the networks begin to count: 801 rows of 128256 with 64 95.  Few rows are two
 * launches' latency: one row of 128256 with five alternatives 10.8, 64 rows with none 12, with 20 20.  A bar of the
 * workgroup's own for the alternatives, from what its waves have seen, took 23 of 128 us off 801 rows with 64; the registers
 * without a passing logit skipped one by one 20 of 123 off 4001 rows of 25001 with five.
 *
 * exp((l - m) / T) is taken as exp2((l - m) * (log2 e / T)): one rounding of the product, 2^-24 |l - m| / T relative.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_serve_device.h"

namespace wsr_serve {

constexpr int LT = 256, LW = LT / WAVE;       /* threads, waves */
typedef uint64_t key64;

struct LogStat {
    float m, s, e;                            /* largest logit; sums of 2^x and of x 2^x, x = (l - m) log2 e / T */
    float mine;                               /* the given token's logit, and whether there is one; logits before it */
    int32_t ranked, before;
};
struct LogPlan {
    int32_t parts, chunks;                    /* of a row */
    key64* keys;                              /* [n_rows][parts][n_top] */
    LogStat* stats;                           /* [n_rows][parts] */
};

/* NaN counts as -inf. */
__device__ __forceinline__ float no_nan(float v) { return fmaxf(v, NEG_INF); }
__device__ __forceinline__ key64 key_of(float v, int i) {
    const uint32_t b = __float_as_uint(v + 0.f);                /* -0 is 0 */
    return (key64)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - (uint32_t)i);
}
__device__ __forceinline__ float logit_of(key64 k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int index_of(key64 k) { return (int)(0xffffffffu - (uint32_t)k); }

__device__ __forceinline__ float temperature_of(const wsr_logprobs& p, int64_t r) {
    const float t = p.temperature ? p.temperature[r] : 1.f;
    return t > 0.f ? fminf(fmaxf(t, 0x1p-126f), 1e30f) : 0.f;   /* log2 e / T is finite */
}
__device__ __forceinline__ float factor_of(float t) { return t > 0.f ? LOG2E / t : 0.f; }

/* s, e against m, moved to the maximum `to` >= m. */
__device__ __forceinline__ void move_max(float& m, float& s, float& e, float to, float k) {
    if (m == to) return;
    const float x = (m - to) * k, f = m == NEG_INF ? 0.f : __builtin_amdgcn_exp2f(x);
    e = f > 0.f ? f * fmaf(s, x, e) : 0.f;
    s = f > 0.f ? s * f : 0.f;
    m = to;
}
__device__ __forceinline__ void join_stats(LogStat& a, LogStat b, float k) {
    const float top = fmaxf(a.m, b.m);
    move_max(a.m, a.s, a.e, top, k);
    move_max(b.m, b.s, b.e, top, k);
    a.s += b.s, a.e += b.e, a.before += b.before;
}

/* ---- sorting networks over a wave: one key per lane ---------------------------------------------------- */

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
/* The value of lane i ^ D. */
template <int D>
__device__ __forceinline__ uint32_t other(uint32_t v) {
    if constexpr (D == 1) return moved<wsr::DPP_XOR1>(v);
    else if constexpr (D == 2) return moved<wsr::DPP_XOR2>(v);
    else if constexpr (D == 4) return moved<0x1B>(moved<wsr::DPP_HALF_MIRROR>(v));      /* i ^ 7, then i ^ 3 */
    else if constexpr (D == 8) return moved<0x128>(v);          /* a 16-lane row turned by 8 */
    else {
        const bool upper = threadIdx.x & D;
        if constexpr (D == 16) {
            const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
            return upper ? s[0] : s[1];
        } else {
            const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
            return upper ? s[0] : s[1];
        }
    }
}
template <int D>
__device__ __forceinline__ float other(float v) { return __uint_as_float(other<D>(__float_as_uint(v))); }
template <int D>
__device__ __forceinline__ key64 other(key64 v) { return (key64)other<D>((uint32_t)(v >> 32)) << 32 | other<D>((uint32_t)v); }

/* One level: the larger of the two in the lower lane where `down`. */
template <int D, typename T>
__device__ __forceinline__ T level(T v, bool down, int lane) {
    const T o = other<D>(v);
    return (((lane & D) == 0) == down) == (v > o) ? v : o;
}
/* N lanes each of a bitonic sequence put in falling (rising) order. */
template <int N, typename T>
__device__ __forceinline__ T merged(T v, bool down, int lane) {
    if constexpr (N >= 64) v = level<32>(v, down, lane);
    if constexpr (N >= 32) v = level<16>(v, down, lane);
    if constexpr (N >= 16) v = level<8>(v, down, lane);
    if constexpr (N >= 8) v = level<4>(v, down, lane);
    if constexpr (N >= 4) v = level<2>(v, down, lane);
    return level<1>(v, down, lane);
}
/* Whether group lane / N of the wave is an even one; of the whole wave, `last`. */
template <int N>
__device__ __forceinline__ bool even(int lane, bool last) { return N >= WAVE ? last : (lane & N) == 0; }
/* Groups of W lanes put in falling order where they are even, rising where odd; the whole wave falling where `last`. */
template <int W, typename T>
__device__ __forceinline__ T sorted(T v, bool last, int lane) {
    if constexpr (W >= 2) v = merged<2>(v, even<2>(lane, last), lane);
    if constexpr (W >= 4) v = merged<4>(v, even<4>(lane, last), lane);
    if constexpr (W >= 8) v = merged<8>(v, even<8>(lane, last), lane);
    if constexpr (W >= 16) v = merged<16>(v, even<16>(lane, last), lane);
    if constexpr (W >= 32) v = merged<32>(v, even<32>(lane, last), lane);
    if constexpr (W >= 64) v = merged<64>(v, last, lane);
    return v;
}
/* The W largest of the wave, from groups that sorted() put in order: in every group, falling where `last`, else rising. */
template <int W, int D = W, typename T>
__device__ __forceinline__ T largest(T v, bool last, int lane) {
    if constexpr (D >= WAVE) return v;
    else {
        v = std::max(v, other<D>(v));
        if constexpr (W > 1) v = merged<W>(v, even<2 * D>(lane, last), lane);
        return largest<W, 2 * D>(v, last, lane);
    }
}
/* The W largest of `count` falling lists of W, in every group, falling.  at(i, j): entry j of list i (0 past the lists). */
template <int W, int STEP, typename F>
__device__ __forceinline__ key64 largest_of(int count, int lane, const F& at) {
    constexpr int G = WAVE / W, AHEAD = 4;
    const int g = lane / W, j = lane % W;
    const bool down = even<W>(lane, true);
    key64 best = 0;
    for (int i0 = 0; i0 < count; i0 += AHEAD * G * STEP) {
        key64 o[AHEAD];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) o[a] = at(i0 + (a * G + g) * STEP, down ? W - 1 - j : j);
#pragma unroll
        for (int a = 0; a < AHEAD; ++a)
            if (i0 + a * G * STEP < count) {
                best = std::max(best, o[a]);
                if constexpr (W > 1) best = merged<W>(best, down, lane);
            }
    }
    return largest<W>(best, true, lane);
}
__device__ __forceinline__ key64 lane_key(key64 v, int lane) {
    return (key64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

constexpr int ROOM = 5 * WAVE;                /* up to 63 that wait and four of each lane */

/* The best W of a wave, and what waits to be merged into it. */
template <int W>
struct Best {
    key64 best, least;                        /* this lane's, falling in every group of W; the n-th, which others have to pass */
    float bar;                                /* its logit, -inf at the start */
    int waiting, n;
    key64* room;                              /* [ROOM] in LDS */

    __device__ __forceinline__ void init(key64* lds, int n_top) { best = 0, least = 0, bar = NEG_INF, waiting = 0, n = n_top, room = lds; }
    __device__ __forceinline__ void raise(key64 k) {
        if (k > least) least = k, bar = logit_of(k);
    }
    __device__ __forceinline__ void merge(key64 v, int lane) {
        const key64 r = largest<W>(sorted<W>(v, false, lane), false, lane);
        best = merged<W>(std::max(best, r), true, lane);
        raise(lane_key(best, n - 1));
    }
    /* Keys that pass `least` (or are it) of all lanes wait in the room, ... */
    __device__ __forceinline__ void add(key64 v, bool in, int lane) {
        const uint64_t who = __ballot(in && v >= least);
        if (who >> lane & 1) room[waiting + __builtin_popcountll(who & ((1ull << lane) - 1))] = v;
        waiting += __builtin_popcountll(who);
    }
    /* ... and are merged, the last 64 at a time. */
    __device__ __forceinline__ bool drain(int lane) {
        const bool any = waiting >= WAVE;
#pragma unroll 1
        while (waiting >= WAVE) {
            waiting -= WAVE;
            wave_fence();
            merge(room[waiting + lane], lane);
        }
        return any;
    }
    __device__ __forceinline__ void flush(int lane) {
        drain(lane);
        wave_fence();
        if (waiting) merge(lane < waiting ? room[lane] : 0, lane);
        waiting = 0;
        wave_fence();
    }
};

/* What is stored for a row, by one wave: its statistics and best keys. */
__device__ __forceinline__ void finish(const wsr_logprobs& p, int64_t r, float t, const LogStat& st, key64 best, int lane) {
    const float log_s = logf(st.s);
    auto log_prob = [&](float l, bool first) {
        if (!(l > NEG_INF)) return NEG_INF;
        if (t == 0.f) return first ? 0.f : NEG_INF;
        return (l == st.m ? 0.f : (l - st.m) / t) - log_s;
    };
    if (lane < p.n_top) {
        p.top[r * p.n_top + lane] = best ? index_of(best) : -1;
        if (p.top_logp) p.top_logp[r * p.n_top + lane] = best ? log_prob(logit_of(best), lane == 0) : NEG_INF;
    }
    if (lane) return;
    if (p.logp) p.logp[r] = st.ranked ? log_prob(st.mine, st.before == 0) : NEG_INF;
    if (p.rank) p.rank[r] = st.ranked ? st.before : -1;
    if (p.entropy) p.entropy[r] = t == 0.f || st.m == NEG_INF ? 0.f : fmaxf(log_s - 0.6931471805599453f * (st.e / st.s), 0.f);
}

/* What the waves of a workgroup show each other without a barrier. */
__device__ __forceinline__ float seen(const float* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void show(float* at, float v) { __hip_atomic_store(at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

/* TOP: no alternatives, one, or up to 8, 32 or 64.  VU: 16-byte loads per thread of a chunk. */
template <int VU, int TOP>
__global__ __launch_bounds__(LT) __attribute__((amdgpu_waves_per_eu(6))) void k_logprobs(wsr_logprobs p, LogPlan pl) {
    constexpr int CHUNK = LT * VU * 4;
    __shared__ key64 room[TOP > 1 ? LW : 1][ROOM];
    __shared__ key64 lists[LW][TOP > 0 ? TOP : 1];
    __shared__ LogStat sums[LW];
    __shared__ float quarter[LW];                               /* the n / 4-th largest logit that each wave has seen */
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), n = (int)p.vocab;
    const int64_t r = blockIdx.x / (uint32_t)pl.parts;
    const int part = (int)(blockIdx.x % (uint32_t)pl.parts);
    const int begin = part * pl.chunks / pl.parts, end = (part + 1) * pl.chunks / pl.parts;
    const float* row = (const float*)((const char*)p.logits + r * p.row_stride);
    const int token = p.tokens ? p.tokens[r] : -1;
    const float t = temperature_of(p, r);
    float next[VU][4];
    auto load = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int i = chunk * CHUNK + (u * LT + (int)threadIdx.x) * 4;
            if (i + 4 <= n) {
                /* read once: 2055 rows of 50257 87.8 us without the hint, so 81 */
                const f4_t q = __builtin_nontemporal_load((const wsr_step::f4_any_t*)(row + i));
#pragma unroll
                for (int j = 0; j < 4; ++j) next[u][j] = q[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) next[u][j] = i + j < n ? row[i + j] : NEG_INF;
            }
        }
    };
    load(begin);
    const float k = factor_of(t);
    const bool ranked = token >= 0 && token < n;
    const float mine = ranked ? no_nan(row[token]) : __builtin_inff();
    const int fourth = (p.n_top + LW - 1) / LW - 1;
    float m = NEG_INF, s = 0.f, e = 0.f, one = NEG_INF;
    int before = 0, one_at = 0x7fffffff;
    Best<(TOP > 1 ? TOP : 2)> b;
    if constexpr (TOP > 1) b.init(room[wave], p.n_top);
#pragma unroll 1
    for (int c = begin; c < end; ++c) {
        float v[VU][4];
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) v[u][j] = no_nan(next[u][j]);
        if (c + 1 < end) load(c + 1);
        const int i0 = c * CHUNK + (int)threadIdx.x * 4;
        float top = v[0][0];
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, v[u][j]);
        if (top > m) move_max(m, s, e, top, k);
        if (__ballot(m == __builtin_inff())) {
#pragma unroll
            for (int u = 0; u < VU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = v[u][j] == m ? 0.f : fmaxf((v[u][j] - m) * k, -200.f), f = v[u][j] > NEG_INF ? __builtin_amdgcn_exp2f(x) : 0.f;
                    s += f;
                    e = fmaf(f, x, e);
                }
        } else {
            /* -inf gives 2^-200, which is 0, and 0 times -200 */
            const float base = m == NEG_INF ? 0.f : m;
#pragma unroll
            for (int u = 0; u < VU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = fmaxf((v[u][j] - base) * k, -200.f), f = __builtin_amdgcn_exp2f(x);
                    s += f;
                    e = fmaf(f, x, e);
                }
        }
        /* logits before the given token come before it where they equal its, those behind it do not */
        if (c * CHUNK + CHUNK <= token) {
#pragma unroll
            for (int u = 0; u < VU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) before += __builtin_popcountll(__ballot(v[u][j] >= mine));
        } else if (c * CHUNK > token) {
#pragma unroll
            for (int u = 0; u < VU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) before += __builtin_popcountll(__ballot(v[u][j] > mine));
        } else {
#pragma unroll
            for (int u = 0; u < VU; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    before += __builtin_popcountll(__ballot(v[u][j] > mine || (v[u][j] == mine && i0 + u * LT * 4 + j < token)));
        }
        if constexpr (TOP == 1) {
            if (__ballot(top > one))
#pragma unroll
                for (int u = 0; u < VU; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (v[u][j] > one) one = v[u][j], one_at = i0 + u * LT * 4 + j;
        }
        if constexpr (TOP > 1) {
            /* again for the second chunk: 1461 rows of 32000 with 21 46.3 us, so 44.9; for the third too, no less */
            if (c < begin + 2) {
                const int order = __builtin_bit_cast(int, sorted<WAVE>(m, true, lane));
                const float bar = __builtin_bit_cast(float, __builtin_amdgcn_readlane(order, p.n_top - 1));
                if (bar > NEG_INF) b.raise(key_of(bar, -1));
                if (lane == 0) show(&quarter[wave], __builtin_bit_cast(float, __builtin_amdgcn_readlane(order, fourth)));
                if (c == begin) __syncthreads();
            }
            /* four waves that have seen n / 4 logits of at least this: no smaller one is among the workgroup's n.  The waves
               write theirs at any time: whichever of a wave's values is read, it has seen n / 4 logits of at least that, so that
               the results do not depend on it. */
            float common = seen(&quarter[0]);
#pragma unroll
            for (int w = 1; w < LW; ++w) common = fminf(common, seen(&quarter[w]));
            if (common > b.bar) b.raise(key_of(common, -1));
            if (__ballot(top >= b.bar && top > NEG_INF))
#pragma unroll
                for (int u = 0; u < VU; ++u) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (__ballot(v[u][j] >= b.bar)) b.add(key_of(v[u][j], i0 + u * LT * 4 + j), v[u][j] > NEG_INF, lane);
                    if (b.drain(lane) && lane == fourth) show(&quarter[wave], logit_of(b.best));
                }
        }
    }
    /* a wave's results, then the workgroup's */
    move_max(m, s, e, wsr_step::wave_max(m), k);
    s = wsr::wave_sum(s), e = wsr::wave_sum(e);
    if constexpr (TOP == 1) {
        const float top = wsr_step::wave_max(one);
        const int where = wsr_step::wave_min(one == top ? one_at : 0x7fffffff);
        if (lane == 0) lists[wave][0] = top > NEG_INF ? key_of(top, where) : 0;
    }
    if constexpr (TOP > 1) {
        b.flush(lane);
        if (lane < TOP) lists[wave][lane] = b.best;
    }
    if (lane == 0) sums[wave] = LogStat{m, s, e, mine, ranked, before};
    __syncthreads();
    if (wave) return;
    LogStat st = sums[0];
    for (int w = 1; w < LW; ++w) join_stats(st, sums[w], k);
    key64 best = 0;
    if constexpr (TOP > 0) best = largest_of<TOP, 1>(LW, lane, [&](int i, int j) { return i < LW ? lists[i][j] : 0; });
    if (pl.parts == 1) {
        finish(p, r, t, st, best, lane);
    } else {
        if (TOP && lane < p.n_top) pl.keys[(int64_t)blockIdx.x * p.n_top + lane] = best;
        if (lane == 0) pl.stats[blockIdx.x] = st;
    }
}

/* A row's parts; a wave takes every fourth. */
template <int TOP>
__global__ __launch_bounds__(LT) void k_logprobs_join(wsr_logprobs p, LogPlan pl) {
    __shared__ key64 lists[LW][TOP > 0 ? TOP : 1];
    __shared__ LogStat sums[LW];
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), parts = pl.parts;
    const int64_t r = blockIdx.x, at = r * parts;
    const float t = temperature_of(p, r), k = factor_of(t);
    LogStat st = pl.stats[at];
    if (threadIdx.x) st.m = NEG_INF, st.s = 0.f, st.e = 0.f, st.before = 0;
    for (int i = threadIdx.x ? threadIdx.x : LT; i < parts; i += LT) join_stats(st, pl.stats[at + i], k);
    key64 best = 0;
    if constexpr (TOP > 0)
        best = largest_of<TOP, LW>(parts - wave, lane, [&](int i, int j) {
            return i + wave < parts && j < p.n_top ? pl.keys[(at + i + wave) * p.n_top + j] : 0;
        });
    move_max(st.m, st.s, st.e, wsr_step::wave_max(st.m), k);
    st.s = wsr::wave_sum(st.s), st.e = wsr::wave_sum(st.e);
#pragma unroll
    for (int d = 32; d; d >>= 1) st.before += __shfl_xor(st.before, d);
    if (lane == 0) sums[wave] = st;
    if (TOP > 0 && lane < TOP) lists[wave][lane] = best;
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < LW; ++w) join_stats(st, sums[w], k);
    if constexpr (TOP > 0) best = largest_of<TOP, 1>(LW, lane, [&](int i, int j) { return i < LW ? lists[i][j] : 0; });
    finish(p, r, t, st, best, lane);
}

/* ---- host ------------------------------------------------------------------------------------------ */

constexpr int VU = 4, CHUNK = LT * VU * 4;
constexpr int HELD = 1536;                    /* workgroups that the chip holds: six waves per SIMD */
static size_t key_bytes(int64_t items, int32_t n_top) { return (items * n_top * sizeof(key64) + 255) / 256 * 256; }
/* Rows are cut into parts of four chunks or more while those are no more than the chip holds, of eight up to twice as many (801
   rows of 128256 75 us whole, in three parts 71; 1000 rows of 32000 31 whole, in two parts of four chunks 38), and into
   shorter ones where they would be fewer than one for each CU. */
static LogPlan plan_of(const wsr_logprobs& p, void* ws) {
    LogPlan pl;
    const int64_t chunks = (p.vocab + CHUNK - 1) / CHUNK, rows = std::max<int64_t>(1, p.n_rows);
    const int64_t parts = std::max({std::min(chunks / 4, HELD / rows), std::min(chunks / 8, 2 * HELD / rows),
                                    std::min(chunks, (256 + rows - 1) / rows)});
    pl.chunks = (int32_t)chunks;
    pl.parts = (int32_t)std::max<int64_t>(1, parts);
    pl.keys = static_cast<key64*>(ws);
    pl.stats = reinterpret_cast<LogStat*>(static_cast<char*>(ws) + key_bytes(p.n_rows * pl.parts, p.n_top));
    return pl;
}

/* What the call needs, and any of fewer rows, which may have more parts: as many as plan_of() allows at most. */
size_t logprobs_workspace(const wsr_logprobs& p) {
    const int64_t chunks = (p.vocab + CHUNK - 1) / CHUNK;
    if (chunks == 1) return 256;
    const int64_t items = std::max({std::min(p.n_rows * (chunks / 4), (int64_t)HELD), std::min(p.n_rows * (chunks / 8), (int64_t)2 * HELD),
                                    std::min(p.n_rows * chunks, (int64_t)511)});
    return std::max<size_t>(256, key_bytes(items, p.n_top) + items * sizeof(LogStat));
}

template <int TOP>
static hipError_t launch_top(const wsr_logprobs& p, const LogPlan& pl, hipStream_t s) {
    hipLaunchKernelGGL((k_logprobs<VU, TOP>), dim3((unsigned)(p.n_rows * pl.parts)), dim3(LT), 0, s, p, pl);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.parts == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join<TOP>, dim3((unsigned)p.n_rows), dim3(LT), 0, s, p, pl);
    return hipGetLastError();
}

hipError_t launch_logprobs(const wsr_logprobs& p, void* ws, hipStream_t s) {
    const LogPlan pl = plan_of(p, ws);
    return p.n_top == 0 ? launch_top<0>(p, pl, s) : p.n_top == 1 ? launch_top<1>(p, pl, s) : p.n_top <= 8 ? launch_top<8>(p, pl, s)
           : p.n_top <= 32 ? launch_top<32>(p, pl, s) : launch_top<64>(p, pl, s);
}

}  // namespace wsr_serve
