/*
 * wsr_verify.hip - verification of drafted tokens: softmax statistics of every logits row, then the
 * acceptance of each sequence's drafts and the race for its next token.
 *
 *   k_verify_stats   (row, chunk): largest logit, its lowest index and the sum of exponentials, one
 *                    read of the row; chunks of CHUNK logits keep few rows spread over the chip
 *   k_verify_race    (sequence, chunk): joins the row statistics, decides, then w / noise over its
 *                    chunk of the one row that the next token is drawn from
 *   k_verify_finish  (sequence): the best of the chunks
 *
 * Bound by HBM at large batches (the rows once, one row and the noise again), by three launches'
 * latency at small ones.  exp((l - m) / T) is taken as exp2((l - m) * (log2 e / T)): the one rounding
 * of the product costs 2^-24 |l - m| / T relative, below 1e-6 for every token that can matter.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int VT = 256;                       /* threads */
constexpr int VU = 8;                         /* 16-byte loads per thread */
constexpr int CHUNK = VT * VU * 4;
constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f;

struct Stat {
    float m, s;      /* largest logit; sum of exp((l - m) / T) */
    int32_t at;      /* lowest index of m */
    int32_t pad;
};
struct Best {
    float w, p;      /* largest residual score and largest plain score */
    int32_t wi, pi;
};

__device__ __forceinline__ float no_nan(float v) { return v == v ? v : NEG_INF; }
/* exp of a logit against its row's maximum: equal values give 1 whatever they are (+inf included). */
__device__ __forceinline__ float exp_from(float l, float m, float c) {
    return l == m ? 1.f : __builtin_amdgcn_exp2f((l - m) * c);
}

__device__ __forceinline__ float temperature_of(const wsr_verify& p, int b) {
    const float t = p.temperature ? p.temperature[b] : 1.f;
    return t > 0.f ? t : 0.f;
}
/* log2 e / T, the factor of exp2; negative for T = 0, where all probability is on one index. */
__device__ __forceinline__ float factor_of(float t) { return t > 0.f ? LOG2E / t : -1.f; }
__device__ __forceinline__ int count_of(const wsr_verify& p, int b) {
    const int c = p.counts ? p.counts[b] : p.n_drafts;
    return min(max(c, 0), p.n_drafts);
}

/* Row r of a sequence: target rows 0 .. n_drafts, then draft rows; null where the count leaves it out. */
__device__ __forceinline__ const float* row_of(const wsr_verify& p, int b, int r, int count) {
    if (r <= p.n_drafts)
        return r > count ? nullptr : (const float*)((const char*)p.target + b * p.target_seq_stride + r * p.target_row_stride);
    r -= p.n_drafts + 1;
    return r >= count ? nullptr : (const float*)((const char*)p.draft + b * p.draft_seq_stride + r * p.draft_row_stride);
}

/* A thread's VU runs of four elements of a chunk; `fill` past the row's end. */
__device__ __forceinline__ void load_chunk(const float* row, int64_t at, int64_t n, float fill, float (&v)[VU][4]) {
#pragma unroll
    for (int u = 0; u < VU; ++u) {
        const int64_t i = at + (u * VT + threadIdx.x) * 4;
        if (i + 4 <= n) {
            const f4_t q = *(const f4_any_t*)(row + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[u][j] = q[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[u][j] = i + j < n ? row[i + j] : fill;
        }
    }
}

__device__ __forceinline__ void better(float& w, int& i, float w2, int i2) {
    if (w2 > w || (w2 == w && i2 < i)) w = w2, i = i2;
}
__device__ __forceinline__ void wave_best(float& w, int& i) {
#pragma unroll
    for (int k = 32; k; k >>= 1) {
        const float w2 = __shfl_xor(w, k);
        const int i2 = __shfl_xor(i, k);
        better(w, i, w2, i2);
    }
}

__global__ __launch_bounds__(VT) void k_verify_stats(wsr_verify p, Stat* stats, int rows, int chunks) {
    __shared__ float sm[VT / WAVE], ss[VT / WAVE];
    __shared__ int si[VT / WAVE];
    const int c = blockIdx.x % chunks, r = blockIdx.x / chunks % rows, b = blockIdx.x / chunks / rows;
    const float* row = row_of(p, b, r, count_of(p, b));
    if (!row) return;
    float v[VU][4];
    load_chunk(row, (int64_t)c * CHUNK, p.vocab, NEG_INF, v);
    float m = NEG_INF;
    int at = 0x7fffffff;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[u][j] = no_nan(v[u][j]);
            if (v[u][j] > m) m = v[u][j], at = c * CHUNK + (u * VT + (int)threadIdx.x) * 4 + j;
        }
    wave_best(m, at);
    const int wave = threadIdx.x / WAVE;
    if (threadIdx.x % WAVE == 0) sm[wave] = m, si[wave] = at;
    __syncthreads();
    m = sm[0], at = si[0];
#pragma unroll
    for (int w = 1; w < VT / WAVE; ++w) better(m, at, sm[w], si[w]);
    const float k = factor_of(temperature_of(p, b));
    float s = 0.f;
    if (m > NEG_INF)
#pragma unroll
        for (int u = 0; u < VU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) s += v[u][j] > NEG_INF ? exp_from(v[u][j], m, k) : 0.f;
    s = block_sum<VT / WAVE>(s, ss);
    if (threadIdx.x == 0) stats[((int64_t)b * rows + r) * chunks + c] = Stat{m, s, at, 0};
}

/* A row's statistics from its chunks, by one wave. */
__device__ __forceinline__ Stat join_row(const Stat* st, int chunks, float t) {
    const int lane = threadIdx.x % WAVE;
    float m = NEG_INF;
    int at = 0x7fffffff;
    for (int c = lane; c < chunks; c += WAVE) better(m, at, st[c].m, st[c].at);
    wave_best(m, at);
    const float k = factor_of(t);
    float s = 0.f;
    for (int c = lane; c < chunks; c += WAVE)
        if (st[c].m > NEG_INF) s += st[c].s * exp_from(st[c].m, m, k);
    return Stat{m, wsr::wave_sum(s), at, 0};
}

/* The probability of logit l (index i) in a row. */
__device__ __forceinline__ float prob(float l, int i, const Stat& st, float inv, float k) {
    if (k < 0.f) return i == st.at && st.m > NEG_INF ? 1.f : 0.f;
    l = no_nan(l);
    return l > NEG_INF ? exp_from(l, st.m, k) * inv : 0.f;
}

__device__ __forceinline__ float log_prob(float l, int i, const Stat& st, float t) {
    if (t == 0.f) return i == st.at && st.m > NEG_INF ? 0.f : NEG_INF;
    l = no_nan(l);
    if (!(l > NEG_INF)) return NEG_INF;
    return (l == st.m ? 0.f : (l - st.m) / t) - logf(st.s);
}

constexpr int MAX_ROWS = 2 * 63 + 1;

__global__ __launch_bounds__(VT) void k_verify_race(wsr_verify p, const Stat* stats, Best* best, Stat* last, int rows,
                                                    int chunks) {
    __shared__ Stat all[MAX_ROWS];
    __shared__ float sw[VT / WAVE], sp[VT / WAVE];
    __shared__ int swi[VT / WAVE], spi[VT / WAVE], verdict;
    const int c = blockIdx.x % chunks, b = blockIdx.x / chunks, wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    const int count = count_of(p, b), n = p.n_drafts;
    const float t = temperature_of(p, b), k = factor_of(t);
    for (int r = wave; r < rows; r += VT / WAVE) {
        if (!row_of(p, b, r, count)) continue;
        const Stat st = join_row(stats + ((int64_t)b * rows + r) * chunks, chunks, t);
        if (lane == 0) all[r] = st;
    }
    __syncthreads();
    if (wave == 0) {
        /* lane i judges draft i */
        bool pass = false;
        float lp = 0.f;
        if (lane < count) {
            const int x = p.tokens[(int64_t)b * n + lane];
            if (x >= 0 && x < p.vocab) {
                const Stat& st = all[lane];
                const float l = row_of(p, b, lane, count)[x];
                const float px = prob(l, x, st, 1.f / st.s, k);
                float qx = 1.f;
                if (p.draft) {
                    const Stat& sq = all[n + 1 + lane];
                    qx = prob(row_of(p, b, n + 1 + lane, count)[x], x, sq, 1.f / sq.s, k);
                }
                pass = p.uniform[(int64_t)b * n + lane] * qx < px;
                lp = log_prob(l, x, st, t);
            }
        }
        const uint64_t failed = ~__ballot(pass);
        const int accepted = __builtin_ctzll(failed);        /* lane 63 never passes: count <= 63 */
        if (lane == 0) verdict = accepted;
        if (c == 0) {
            for (int i = lane; i <= n; i += WAVE) {
                if (i < accepted) p.out[(int64_t)b * (n + 1) + i] = p.tokens[(int64_t)b * n + i];
                else if (i > accepted) p.out[(int64_t)b * (n + 1) + i] = -1;
                if (p.logp) {
                    if (i < accepted) p.logp[(int64_t)b * (n + 1) + i] = lp;
                    else if (i > accepted) p.logp[(int64_t)b * (n + 1) + i] = 0.f;
                }
            }
            if (lane == 0) p.accepted[b] = accepted, last[b] = all[accepted];
        }
    }
    __syncthreads();
    const int a = verdict;
    const Stat st = all[a];
    const bool residual = a < count;
    const float* prow = row_of(p, b, a, count);
    const float* qrow = residual && p.draft ? row_of(p, b, n + 1 + a, count) : nullptr;
    const Stat sq = qrow ? all[n + 1 + a] : Stat{0.f, 1.f, 0, 0};
    const int x = residual && !p.draft ? p.tokens[(int64_t)b * n + a] : -1;
    const float ip = 1.f / st.s, iq = 1.f / sq.s;
    float v[VU][4], z[VU][4], q[VU][4];
    load_chunk((const float*)((const char*)p.noise + b * p.noise_seq_stride), (int64_t)c * CHUNK, p.vocab, 1.f, z);
    load_chunk(prow, (int64_t)c * CHUNK, p.vocab, NEG_INF, v);
    if (qrow) load_chunk(qrow, (int64_t)c * CHUNK, p.vocab, NEG_INF, q);
    float bw = 0.f, bp = 0.f;
    int bwi = 0x7fffffff, bpi = 0x7fffffff;
#pragma unroll
    for (int u = 0; u < VU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c * CHUNK + (u * VT + (int)threadIdx.x) * 4 + j;
            if (i >= p.vocab) continue;
            const float pv = prob(v[u][j], i, st, ip, k);
            float w = pv;
            if (qrow) w = pv - prob(q[u][j], i, sq, iq, k);
            else if (i == x) w = pv - 1.f;
            const float rn = 1.f / z[u][j];
            if (w > 0.f && w * rn > bw) bw = w * rn, bwi = i;
            if (pv > 0.f && pv * rn > bp) bp = pv * rn, bpi = i;
        }
    wave_best(bw, bwi);
    wave_best(bp, bpi);
    if (lane == 0) sw[wave] = bw, swi[wave] = bwi, sp[wave] = bp, spi[wave] = bpi;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < VT / WAVE; ++w) better(bw, bwi, sw[w], swi[w]), better(bp, bpi, sp[w], spi[w]);
        best[(int64_t)b * chunks + c] = Best{bw, bp, bwi, bpi};
    }
}

__global__ __launch_bounds__(WAVE) void k_verify_finish(wsr_verify p, const Best* best, const Stat* last, int chunks) {
    const int b = blockIdx.x, lane = threadIdx.x;
    float w = 0.f, q = 0.f;
    int wi = 0x7fffffff, qi = 0x7fffffff;
    for (int c = lane; c < chunks; c += WAVE) {
        const Best o = best[(int64_t)b * chunks + c];
        better(w, wi, o.w, o.wi);
        better(q, qi, o.p, o.pi);
    }
    wave_best(w, wi);
    wave_best(q, qi);
    if (lane) return;
    const int token = w > 0.f ? wi : q > 0.f ? qi : -1;
    const int a = p.accepted[b];
    const int64_t at = (int64_t)b * (p.n_drafts + 1) + a;
    p.out[at] = token;
    if (p.logp) p.logp[at] = token < 0 ? NEG_INF : log_prob(row_of(p, b, a, a)[token], token, last[b], temperature_of(p, b));
}

struct VerifyPlan {
    int rows, chunks;
    size_t best_at, last_at, bytes;
};
static VerifyPlan plan_of(const wsr_verify& p) {
    VerifyPlan v;
    v.rows = p.n_drafts + 1 + (p.draft ? p.n_drafts : 0);
    v.chunks = (int)((p.vocab + CHUNK - 1) / CHUNK);
    const size_t pairs = (size_t)p.n_seqs * v.chunks;
    v.best_at = (pairs * v.rows * sizeof(Stat) + 255) / 256 * 256;
    v.last_at = v.best_at + (pairs * sizeof(Best) + 255) / 256 * 256;
    v.bytes = v.last_at + (size_t)p.n_seqs * sizeof(Stat);
    return v;
}

size_t verify_workspace(const wsr_verify& p) { return plan_of(p).bytes; }

hipError_t launch_verify(const wsr_verify& p, void* ws, hipStream_t s) {
    const VerifyPlan v = plan_of(p);
    Stat* stats = static_cast<Stat*>(ws);
    Best* best = reinterpret_cast<Best*>(static_cast<char*>(ws) + v.best_at);
    Stat* last = reinterpret_cast<Stat*>(static_cast<char*>(ws) + v.last_at);
    const int64_t blocks = (int64_t)p.n_seqs * v.rows * v.chunks;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL(k_verify_stats, dim3((unsigned)blocks), dim3(VT), 0, s, p, stats, v.rows, v.chunks);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_verify_race, dim3((unsigned)(p.n_seqs * v.chunks)), dim3(VT), 0, s, p, stats, best, last, v.rows,
                       v.chunks);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(k_verify_finish, dim3((unsigned)p.n_seqs), dim3(WAVE), 0, s, p, best, last, v.chunks);
    return hipGetLastError();
}

}  // namespace wsr_step
