/*
 * wsr_logprobs.hip - log probabilities of given tokens, with rank, entropy and the most likely alternatives.
 *
 *   p = softmax(l / T):  log p_x = (l_x - m) / T - log s,  s = sum exp((l - m) / T),
 *   entropy = log s + sum p (m - l) / T
 *
 * One read of a row: every lane keeps a maximum of its own, the two sums against it, and how many logits come before the
 * given token's.  A row is a workgroup's, or, where rows are few, several parts' that a second launch joins.
 *
 * The n largest: a wave keeps its best 64 in order, one per lane, as 64-bit keys (the logit's bits in an order of whole
 * numbers, then the index from the top, so that equal logits go by index).  Logits that pass the n-th key, which after
 * the first few hundred are rare, are collected in LDS and merged in 64 at a time, sorted by compare-and-swap networks
 * over the wave.  The first chunk's threshold is the n-th largest of the lanes' maxima, which n logits reach.
 *
 * exp((l - m) / T) is taken as exp2((l - m) * (log2 e / T)): one rounding of the product, 2^-24 |l - m| / T relative.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_serve_device.h"

namespace wsr_serve {

constexpr int LT = 256, LW = LT / WAVE;       /* threads, waves */
typedef uint64_t key64;

struct LogPlan {
    int32_t parts, per;                       /* of a row, and chunks of a part */
    key64* keys;                              /* [n_rows][parts][n_top] */
    struct LogStat* stats;                    /* [n_rows][parts] */
};
struct LogStat {
    float m, s, e;                            /* largest logit; sums of 2^x and of x 2^x, x = (l - m) log2 e / T */
    int32_t before;
};

__device__ __forceinline__ float no_nan(float v) { return v == v ? v + 0.f : NEG_INF; }     /* and -0 is 0 */
__device__ __forceinline__ key64 key_of(float v, int i) {
    const uint32_t b = __float_as_uint(v);
    return (key64)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - (uint32_t)i);
}
__device__ __forceinline__ float logit_of(key64 k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int index_of(key64 k) { return (int)(0xffffffffu - (uint32_t)k); }

__device__ __forceinline__ float temperature_of(const wsr_logprobs& p, int64_t r) {
    const float t = p.temperature ? p.temperature[r] : 1.f;
    return t > 0.f ? fminf(t, 1e30f) : 0.f;
}

/* s, e against m, moved to the maximum `to` >= m. */
__device__ __forceinline__ void move_max(float& m, float& s, float& e, float to, float k) {
    if (m == to) return;
    const float x = (m - to) * k, f = m == NEG_INF ? 0.f : __builtin_amdgcn_exp2f(x);
    e = f > 0.f ? f * fmaf(s, x, e) : 0.f;
    s = f > 0.f ? s * f : 0.f;
    m = to;
}

__device__ __forceinline__ key64 shfl_xor(key64 v, int d) { return __shfl_xor((unsigned long long)v, d); }
__device__ __forceinline__ key64 lane_key(key64 v, int lane) {
    return (key64)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

/* One level of a sorting network: the larger of the two in the lower lane where `down`. */
__device__ __forceinline__ key64 level(key64 v, int d, bool down, int lane) {
    const key64 o = shfl_xor(v, d);
    return (((lane & d) == 0) == down) == (v > o) ? v : o;
}
/* A bitonic sequence put in falling order. */
__device__ __forceinline__ key64 fall(key64 v, int lane) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = level(v, d, true, lane);
    return v;
}
/* Rising (falling) order over the wave. */
template <bool DOWN>
__device__ __forceinline__ key64 sorted(key64 v, int lane) {
#pragma unroll
    for (int n = 2; n <= WAVE; n <<= 1)
#pragma unroll
        for (int d = n / 2; d; d >>= 1) v = level(v, d, n == WAVE ? DOWN : ((lane & n) == 0) == DOWN, lane);
    return v;
}

/* The wave's LDS stores are there for its loads that follow. */
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }

constexpr int ROOM = 9 * WAVE;                /* up to 63 that wait and eight of each lane */

/* The best of a wave, and what waits to be merged into it. */
struct Best {
    key64 best, least;                        /* this lane's; the n-th, which others have to pass */
    float bar;                                /* its logit, -inf at the start */
    int waiting, n;
    key64* room;                              /* [ROOM] in LDS */

    __device__ __forceinline__ void init(key64* lds, int n_top) { best = 0, least = 0, bar = NEG_INF, waiting = 0, n = n_top, room = lds; }
    __device__ __forceinline__ void raise(key64 k) {
        if (k > least) least = k, bar = logit_of(k);
    }
    __device__ __forceinline__ void merge(key64 v, int lane) {
        const key64 r = sorted<false>(v, lane);
        best = fall(best > r ? best : r, lane);
        raise(lane_key(best, n - 1));
    }
    /* Keys that pass `least` (or are it) of all lanes wait in the room, ... */
    __device__ __forceinline__ void add(key64 v, bool in, int lane) {
        const uint64_t who = __ballot(in && v >= least);
        if (who >> lane & 1) room[waiting + __builtin_popcountll(who & ((1ull << lane) - 1))] = v;
        waiting += __builtin_popcountll(who);
    }
    /* ... and are merged, the last 64 at a time. */
    __device__ __forceinline__ void drain(int lane) {
#pragma unroll 1
        while (waiting >= WAVE) {
            waiting -= WAVE;
            wave_fence();
            merge(room[waiting + lane], lane);
        }
    }
    __device__ __forceinline__ void flush(int lane) {
        drain(lane);
        wave_fence();
        if (waiting) merge(lane < waiting ? room[lane] : 0, lane);
        waiting = 0;
    }
};

/* What is stored for a row, by one wave: its statistics and best keys. */
__device__ __forceinline__ void finish(const wsr_logprobs& p, int64_t r, const LogStat& st, key64 best, int lane) {
    const float t = temperature_of(p, r), log_s = logf(st.s);
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
    if (p.entropy) p.entropy[r] = t == 0.f || st.m == NEG_INF ? 0.f : fmaxf(log_s - 0.6931471805599453f * (st.e / st.s), 0.f);
    if (p.tokens) {
        const int x = p.tokens[r];
        const bool in = x >= 0 && x < p.vocab;
        const float l = in ? no_nan(((const float*)((const char*)p.logits + r * p.row_stride))[x]) : NEG_INF;
        if (p.logp) p.logp[r] = log_prob(l, st.before == 0);
        if (p.rank) p.rank[r] = in ? st.before : -1;
    }
}

/* TOP: whether alternatives are asked for. */
template <int VU, bool TOP>                   /* VU: 16-byte loads per thread, even */
__global__ __launch_bounds__(LT) void k_logprobs(wsr_logprobs p, LogPlan pl) {
    constexpr int CHUNK = LT * VU * 4;
    __shared__ key64 room[LW][ROOM];
    __shared__ LogStat sums[LW];
    const int64_t r = blockIdx.x / pl.parts;
    const int part = blockIdx.x % pl.parts, lane = threadIdx.x % WAVE, wave = wsr::wave_in_block();
    const float* row = (const float*)((const char*)p.logits + r * p.row_stride);
    const int n = (int)p.vocab, from = part * pl.per * CHUNK, to = (int)std::min<int64_t>((int64_t)from + (int64_t)pl.per * CHUNK, n);
    const float t = temperature_of(p, r), k = t > 0.f ? LOG2E / t : 0.f;
    const int token = p.tokens ? p.tokens[r] : -1;
    const bool ranked = token >= 0 && token < n;
    const float mine = ranked ? no_nan(row[token]) : 0.f;
    float m = NEG_INF, s = 0.f, e = 0.f;
    int before = 0;
    Best b;
    b.init(room[wave], p.n_top);
    auto load = [&](int at, float (&v)[VU][4]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int i = at + (u * LT + (int)threadIdx.x) * 4;
            if (i + 4 <= to) {
                const f4_t q = *(const wsr_step::f4_any_t*)(row + i);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[u][j] = no_nan(q[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[u][j] = i + j < to ? no_nan(row[i + j]) : NEG_INF;
            }
        }
    };
    for (int at = from; at < to; at += CHUNK) {
        float v[VU][4];
        load(at, v);
        const int i0 = at + (int)threadIdx.x * 4;
        float top = v[0][0];
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, v[u][j]);
        if (top > m) move_max(m, s, e, top, k);
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float l = v[u][j], x = l == m ? 0.f : (l - m) * k, f = __builtin_amdgcn_exp2f(x);
                s += l > NEG_INF ? f : 0.f;
                e += l > NEG_INF && f > 0.f ? f * x : 0.f;
                before += l > mine || (l == mine && i0 + u * LT * 4 + j < token);
            }
        if constexpr (TOP) {
            if (at == from) {
                /* the first of a lane's that has its largest, so that equal logits raise no bar above themselves */
                key64 first = 0;
#pragma unroll
                for (int u = 0; u < VU; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (v[u][j] > NEG_INF) first = std::max(first, key_of(v[u][j], i0 + u * LT * 4 + j));
                b.raise(lane_key(sorted<true>(first, lane), b.n - 1));
            }
            if (__ballot(top >= b.bar && top > NEG_INF))
#pragma unroll
                for (int u = 0; u < VU; ++u) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) b.add(key_of(v[u][j], i0 + u * LT * 4 + j), v[u][j] > NEG_INF, lane);
                    if (u % 2) b.drain(lane);
                }
        }
    }
    /* a wave's, then the workgroup's */
    const float wm = wsr_step::wave_max(m);
    move_max(m, s, e, wm, k);
    s = wsr::wave_sum(s), e = wsr::wave_sum(e);
#pragma unroll
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
    if constexpr (TOP) {
        b.flush(lane);
        wave_fence();
        room[wave][lane] = b.best;
    }
    if (lane == 0) sums[wave] = LogStat{m, s, e, before};
    __syncthreads();
    if (wave) return;
    LogStat st = sums[0];
    for (int w = 1; w < LW; ++w) {
        LogStat o = sums[w];
        const float top = fmaxf(st.m, o.m);
        move_max(st.m, st.s, st.e, top, k);
        move_max(o.m, o.s, o.e, top, k);
        st.s += o.s, st.e += o.e, st.before += o.before;
    }
    if constexpr (TOP)
#pragma unroll
        for (int w = 1; w < LW; ++w) {
            const key64 o = room[w][WAVE - 1 - lane];
            b.best = fall(b.best > o ? b.best : o, lane);
        }
    if (pl.parts == 1) {
        finish(p, r, st, b.best, lane);
    } else {
        const int64_t at = r * pl.parts + part;
        if (TOP && lane < p.n_top) pl.keys[at * p.n_top + lane] = b.best;
        if (lane == 0) pl.stats[at] = st;
    }
}

/* A row's parts, by one wave. */
__global__ __launch_bounds__(WAVE) void k_logprobs_join(wsr_logprobs p, LogPlan pl) {
    __shared__ key64 room[2 * WAVE];      /* one key of each lane at a time */
    const int64_t r = blockIdx.x;
    const int lane = threadIdx.x;
    const float t = temperature_of(p, r), k = t > 0.f ? LOG2E / t : 0.f;
    LogStat st{NEG_INF, 0.f, 0.f, 0};
    for (int c = lane; c < pl.parts; c += WAVE) {
        LogStat o = pl.stats[r * pl.parts + c];
        const float top = fmaxf(st.m, o.m);
        move_max(st.m, st.s, st.e, top, k);
        move_max(o.m, o.s, o.e, top, k);
        st.s += o.s, st.e += o.e, st.before += o.before;
    }
    move_max(st.m, st.s, st.e, wsr_step::wave_max(st.m), k);
    st.s = wsr::wave_sum(st.s), st.e = wsr::wave_sum(st.e);
#pragma unroll
    for (int d = 32; d; d >>= 1) st.before += __shfl_xor(st.before, d);
    Best b;
    b.init(room, p.n_top);
    const key64* keys = pl.keys + r * pl.parts * p.n_top;
    const int all = pl.parts * p.n_top;
    for (int i = 0; i < all; i += WAVE) {
        const key64 v = i + lane < all ? keys[i + lane] : 0;
        b.add(v, v != 0, lane);
        b.drain(lane);
    }
    b.flush(lane);
    finish(p, r, st, b.best, lane);
}

/* ---- host ------------------------------------------------------------------------------------------ */

constexpr int VU = 4;

static LogPlan plan_of(const wsr_logprobs& p, void* ws, size_t* bytes) {
    LogPlan pl;
    const int64_t chunks = (p.vocab + LT * VU * 4 - 1) / (LT * VU * 4);
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(chunks, 2048 / std::max<int64_t>(1, p.n_rows)));
    pl.per = (int32_t)((chunks + want - 1) / want);
    pl.parts = (int32_t)((chunks + pl.per - 1) / pl.per);
    const size_t items = (size_t)p.n_rows * pl.parts, keys = (items * p.n_top * sizeof(key64) + 255) / 256 * 256;
    if (bytes) *bytes = pl.parts == 1 ? 256 : keys + items * sizeof(LogStat);
    pl.keys = static_cast<key64*>(ws);
    pl.stats = reinterpret_cast<LogStat*>(static_cast<char*>(ws) + keys);
    return pl;
}

size_t logprobs_workspace(const wsr_logprobs& p) {
    size_t n;
    plan_of(p, nullptr, &n);
    return n;
}

hipError_t launch_logprobs(const wsr_logprobs& p, void* ws, hipStream_t s) {
    const LogPlan pl = plan_of(p, ws, nullptr);
    const dim3 grid((unsigned)(p.n_rows * pl.parts)), threads(LT);
    if (p.n_top) hipLaunchKernelGGL((k_logprobs<VU, true>), grid, threads, 0, s, p, pl);
    else hipLaunchKernelGGL((k_logprobs<VU, false>), grid, threads, 0, s, p, pl);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || pl.parts == 1) return e;
    hipLaunchKernelGGL(k_logprobs_join, dim3((unsigned)p.n_rows), dim3(WAVE), 0, s, p, pl);
    return hipGetLastError();
}

}  // namespace wsr_serve
