/*
 * wsr_verify.hip - verification of drafted tokens: softmax statistics of every logits row, then the
 * acceptance of each sequence's drafts and the race for its next token.
 *
 *   k_verify_stats   (row, chunk): largest logit, its lowest index and the sum of exponentials, one
 *                    read of the row; chunks keep few rows spread over the chip
 *   k_verify_race    (sequence, chunk): joins the row statistics, decides, then w / noise over its
 *                    chunk of the one row that the next token is drawn from; the last workgroup of a
 *                    sequence to finish takes the best of its chunks (a maximum, so their order is free)
 *
 * Bound by HBM at large batches (the rows once, one row and the noise again: 64 sequences of 7 drafts over 128256
 * logits, 525 MB, 110 us, of which the first launch, at 6.2 TB/s, takes 78), by two launches' chains of dependent loads
 * at small ones (1 sequence of 4 drafts 12 us).  exp((l - m) / T) is taken as exp2((l - m) * (log2 e / T)): the one
 * rounding of the product costs 2^-24 |l - m| / T relative, below 1e-6 for every token that can matter.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int VT = 256;                       /* threads */
/* VU: 16-byte loads per thread; a chunk is VT * VU * 4 logits */
constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f;

struct Stat {
    float m, s;      /* largest logit; sum of exp((l - m) / T) */
    int32_t at;      /* lowest index of m */
    int32_t pad;
};
struct Best {
    float w;         /* the largest score of a chunk */
    int32_t wi;      /* its index */
    float p;         /* the same of plain scores, without the draft's probabilities */
    int32_t pi;
    float wl, pl;    /* their logits */
};

__device__ __forceinline__ float no_nan(float v) { return v == v ? v : NEG_INF; }
/* exp of a logit against its row's maximum: equal values give 1 whatever they are (+inf included). */
__device__ __forceinline__ float exp_from(float l, float m, float c) {
    return l == m ? 1.f : __builtin_amdgcn_exp2f((l - m) * c);
}

__device__ __forceinline__ float temperature_of(const wsr_verify& p, int b) {
    const float t = p.temperature ? p.temperature[b] : 1.f;
    return t > 0.f ? fminf(t, 1e30f) : 0.f;       /* the factor of an infinite one would meet infinite differences */
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
template <int VU>
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
__device__ __forceinline__ void better(Best& a, const Best& b) {
    if (b.w > a.w || (b.w == a.w && b.wi < a.wi)) a.w = b.w, a.wi = b.wi, a.wl = b.wl;
    if (b.p > a.p || (b.p == a.p && b.pi < a.pi)) a.p = b.p, a.pi = b.pi, a.pl = b.pl;
}
/* The largest w of a wave and the lowest index that has it. */
__device__ __forceinline__ void wave_best(float& w, int& i) {
    const float top = wave_max(w);
    i = wave_min(w == top ? i : 0x7fffffff);
    w = top;
}
/* And what belongs to that index. */
__device__ __forceinline__ void wave_best(float& w, int& i, float& l) {
    const int mine = i;
    wave_best(w, i);
    l = __shfl(l, __builtin_ctzll(__ballot(mine == i)));
}
/* Words that workgroups of different XCDs pass to one another: stored to and loaded from where all of them see
   them, past the caches that they do not share. */
struct Words {
    uint64_t w[3];
};
__device__ __forceinline__ void pass_on(Words* to, const Best& b) {
    const Words o = __builtin_bit_cast(Words, b);
#pragma unroll
    for (int i = 0; i < 3; ++i) __hip_atomic_store(&to->w[i], o.w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Best passed(const Words* from) {
    Words o;
#pragma unroll
    for (int i = 0; i < 3; ++i) o.w[i] = __hip_atomic_load(&from->w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_bit_cast(Best, o);
}

template <int VU>
__global__ __launch_bounds__(VT) void k_verify_stats(wsr_verify p, Stat* stats, uint32_t* done, int rows, int chunks) {
    constexpr int CHUNK = VT * VU * 4;
    __shared__ float sm[VT / WAVE], ss[VT / WAVE];
    __shared__ int si[VT / WAVE];
    const int c = blockIdx.x % chunks, r = blockIdx.x / chunks % rows, b = blockIdx.x / chunks / rows;
    if (c == 0 && r == 0 && threadIdx.x == 0) done[b] = 0;    /* for the race's workgroups to count themselves */
    const float* row = row_of(p, b, r, count_of(p, b));
    if (!row) return;
    float v[VU][4];
    load_chunk<VU>(row, (int64_t)c * CHUNK, p.vocab, NEG_INF, v);
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

/* A row's statistics from its chunks, by sixteen lanes (lane j takes chunks j, j + 16, ...), of more than sixteen
   four loaded at a time (1 sequence of 63 chunks 12.7 us one by one, so 11.9). */
__device__ __forceinline__ Stat join_row(const Stat* st, int chunks, float k, int j) {
    float m = NEG_INF, s = 0.f;
    int at = 0x7fffffff;
    auto add = [&](const Stat& o, bool in) __attribute__((always_inline)) {
        if (in && o.m > m) s = s * (m > NEG_INF ? exp_from(m, o.m, k) : 0.f) + o.s, m = o.m, at = o.at;
        else if (in && o.m > NEG_INF) s += o.s * exp_from(o.m, m, k);
    };
    if (chunks <= 16) {
        if (j < chunks) add(st[j], true);
    } else {
        for (int c = j; c < chunks; c += 64) {
            Stat o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = st[min(c + 16 * e, chunks - 1)];
#pragma unroll
            for (int e = 0; e < 4; ++e) add(o[e], c + 16 * e < chunks);
        }
    }
    const float top = row_max(m);
    at = row_min(m == top ? at : 0x7fffffff);
    return Stat{top, row_sum(m > NEG_INF ? s * exp_from(m, top, k) : 0.f), at, 0};
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

template <int VU>
__global__ __launch_bounds__(VT) void k_verify_race(wsr_verify p, const Stat* stats, Words* best, uint32_t* done, int rows,
                                                    int chunks) {
    constexpr int CHUNK = VT * VU * 4;
    __shared__ Stat all[MAX_ROWS];
    __shared__ Best bests[VT / WAVE];
    __shared__ int verdict, last;
    const int c = blockIdx.x % chunks, b = blockIdx.x / chunks, wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
    const int count = count_of(p, b), n = p.n_drafts;
    const float t = temperature_of(p, b), k = factor_of(t);
    /* what does not wait for the statistics: the noise, and (by the first wave) each draft and its logits */
    float v[VU][4], z[VU][4], q[VU][4];
    load_chunk<VU>((const float*)((const char*)p.noise + b * p.noise_seq_stride), (int64_t)c * CHUNK, p.vocab, 1.f, z);
    int x = -1;
    float u = 0.f, lt = NEG_INF, ld = NEG_INF;
    if (wave == 0 && lane < n) {
        x = p.tokens[(int64_t)b * n + lane];
        u = p.uniform[(int64_t)b * n + lane];
        if (lane >= count) x = -1;
        if (x >= 0 && x < p.vocab) {
            lt = row_of(p, b, lane, count)[x];
            if (p.draft) ld = row_of(p, b, n + 1 + lane, count)[x];
        }
    }
    for (int r = threadIdx.x / 16; r < rows; r += VT / 16) {
        const Stat st = join_row(stats + ((int64_t)b * rows + r) * chunks, chunks, k, threadIdx.x % 16);
        if (threadIdx.x % 16 == 0) all[r] = st;
    }
    __syncthreads();
    if (wave == 0) {
        /* lane i judges draft i */
        bool pass = false;
        float lp = 0.f;
        if (x >= 0 && x < p.vocab) {
            const Stat& st = all[lane];
            const float px = prob(lt, x, st, 1.f / st.s, k);
            float qx = 1.f;
            if (p.draft) qx = prob(ld, x, all[n + 1 + lane], 1.f / all[n + 1 + lane].s, k);
            pass = u * qx < px;
            lp = log_prob(lt, x, st, t);
        }
        const int accepted = __builtin_ctzll(~__ballot(pass));   /* lane 63 never passes: count <= 63 */
        if (lane == 0) verdict = accepted;
        if (c == 0) {
            if (lane <= n && lane != accepted) {
                p.out[(int64_t)b * (n + 1) + lane] = lane < accepted ? x : -1;
                if (p.logp) p.logp[(int64_t)b * (n + 1) + lane] = lane < accepted ? lp : 0.f;
            }
            if (lane == 0) p.accepted[b] = accepted;
        }
    }
    __syncthreads();
    const int a = verdict;
    const Stat st = all[a];
    const bool residual = a < count;
    const float* prow = row_of(p, b, a, count);
    const float* qrow = residual && p.draft ? row_of(p, b, n + 1 + a, count) : nullptr;
    load_chunk<VU>(prow, (int64_t)c * CHUNK, p.vocab, NEG_INF, v);
    if (qrow) load_chunk<VU>(qrow, (int64_t)c * CHUNK, p.vocab, NEG_INF, q);
    const Stat sq = qrow ? all[n + 1 + a] : Stat{0.f, 1.f, 0, 0};
    const int point = residual && !p.draft ? p.tokens[(int64_t)b * n + a] : -1;
    const float ip = 1.f / st.s, iq = 1.f / sq.s;
    float bw = 0.f, bp = 0.f, bwl = 0.f, bpl = 0.f;
    int bwi = 0x7fffffff, bpi = 0x7fffffff;
#pragma unroll
    for (int e = 0; e < VU; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c * CHUNK + (e * VT + (int)threadIdx.x) * 4 + j;
            const float pv = prob(v[e][j], i, st, ip, k);        /* 0 past the row's end */
            float w = pv;
            if (qrow) w = pv - prob(q[e][j], i, sq, iq, k);
            else if (i == point) w = pv - 1.f;
            const float rn = __builtin_amdgcn_rcpf(z[e][j]);
            if (w > 0.f && w * rn > bw) bw = w * rn, bwi = i, bwl = v[e][j];
            if (pv * rn > bp) bp = pv * rn, bpi = i, bpl = v[e][j];
        }
    wave_best(bw, bwi, bwl);
    wave_best(bp, bpi, bpl);
    if (lane == 0) bests[wave] = Best{bw, bwi, bp, bpi, bwl, bpl};
    __syncthreads();
    if (threadIdx.x == 0) {
        Best o = bests[0];
#pragma unroll
        for (int w = 1; w < VT / WAVE; ++w) better(o, bests[w]);
        pass_on(&best[(int64_t)b * chunks + c], o);
        /* Counted once the words above have arrived.  What passes between workgroups are agent-scope atomics alone, which no
           cache of one XCD holds, so this wait is all of a release that matters here; a release and an acquire would
           write back and empty caches besides (64 sequences 110 us, with them 156; 33 of 32000 logits 16.2 and 18.6). */
        wait_stores();
        last = __hip_atomic_fetch_add(&done[b], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)chunks - 1;
    }
    __syncthreads();
    if (!last || wave) return;
    Best o{0.f, 0x7fffffff, 0.f, 0x7fffffff, 0.f, 0.f};
    for (int i = lane; i < chunks; i += WAVE) better(o, passed(&best[(int64_t)b * chunks + i]));
    wave_best(o.w, o.wi, o.wl);
    wave_best(o.p, o.pi, o.pl);
    if (lane) return;
    const int token = o.w > 0.f ? o.wi : o.p > 0.f ? o.pi : -1;
    p.out[(int64_t)b * (n + 1) + a] = token;
    if (p.logp) p.logp[(int64_t)b * (n + 1) + a] = token < 0 ? NEG_INF : log_prob(o.w > 0.f ? o.wl : o.pl, token, st, t);
}

struct VerifyPlan {
    int rows, chunks;
    bool fine;
    size_t best_at, done_at, bytes;
};
static VerifyPlan plan_of(const wsr_verify& p) {
    VerifyPlan v;
    v.rows = p.n_drafts + 1 + (p.draft ? p.n_drafts : 0);
    /* chunks of 4096 logits (64 sequences 110 us, with 8192 118, with 2048 173), of 2048 where the former would leave
       most of the chip idle in the race */
    const int64_t wide = (p.vocab + VT * 16 - 1) / (VT * 16);
    v.fine = p.n_seqs * wide < 512;
    v.chunks = (int)(v.fine ? (p.vocab + VT * 8 - 1) / (VT * 8) : wide);
    const size_t pairs = (size_t)p.n_seqs * v.chunks;
    v.best_at = (pairs * v.rows * sizeof(Stat) + 255) / 256 * 256;
    v.done_at = v.best_at + (pairs * sizeof(Words) + 255) / 256 * 256;
    v.bytes = v.done_at + (size_t)p.n_seqs * sizeof(uint32_t);
    return v;
}

size_t verify_workspace(const wsr_verify& p) { return plan_of(p).bytes; }

template <int VU>
static hipError_t launch_two(const wsr_verify& p, const VerifyPlan& v, char* ws, hipStream_t s) {
    Stat* stats = reinterpret_cast<Stat*>(ws);
    Words* best = reinterpret_cast<Words*>(ws + v.best_at);
    uint32_t* done = reinterpret_cast<uint32_t*>(ws + v.done_at);
    hipLaunchKernelGGL(k_verify_stats<VU>, dim3((unsigned)(p.n_seqs * v.rows * v.chunks)), dim3(VT), 0, s, p, stats, done, v.rows,
                       v.chunks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_verify_race<VU>, dim3((unsigned)(p.n_seqs * v.chunks)), dim3(VT), 0, s, p, stats, best, done, v.rows,
                       v.chunks);
    return hipGetLastError();
}

hipError_t launch_verify(const wsr_verify& p, void* ws, hipStream_t s) {
    const VerifyPlan v = plan_of(p);
    /* as many sequences as a launch holds the rows and chunks of, then the next, in the same workspace */
    const int64_t held = most_blocks(VT) / ((int64_t)v.rows * v.chunks);
    for (int64_t b = 0; b < p.n_seqs; b += held) {
        wsr_verify q = p;
        q.n_seqs = (int32_t)std::min<int64_t>(held, p.n_seqs - b);
        q.target = (const float*)((const char*)p.target + b * p.target_seq_stride);
        if (p.draft) q.draft = (const float*)((const char*)p.draft + b * p.draft_seq_stride);
        q.noise = (const float*)((const char*)p.noise + b * p.noise_seq_stride);
        if (p.n_drafts) q.tokens += b * p.n_drafts, q.uniform += b * p.n_drafts;
        if (p.counts) q.counts += b;
        if (p.temperature) q.temperature += b;
        q.out += b * (p.n_drafts + 1), q.accepted += b;
        if (p.logp) q.logp += b * (p.n_drafts + 1);
        const hipError_t e = v.fine ? launch_two<2>(q, v, static_cast<char*>(ws), s) : launch_two<4>(q, v, static_cast<char*>(ws), s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace wsr_step
