/*
 * wsr_append.hip - the projections' fp32 outputs into 16-bit queries, keys and values: norms of each head, rotary
 * positions, and keys and values stored to their pages.
 *
 *   u = norm(x);  (a, b) -> (a cos t - b sin t, b cos t + a sin t),  t = position * frequency
 *
 * Eight values of a head per lane, so that a head of 64, 128 or 256 is 8, 16 or 32 lanes and a wave takes eight, four
 * or two heads at a time.  A lane's values are two runs of four: j .. j + 3 and, rot_dim / 2 on, the other halves of
 * their pairs; past rot_dim, or where pairs stand side by side, eight in a row.  A norm is a sum over the head's lanes.
 * The sine and cosine of a lane's four angles are the same for all heads and taken once per wave: position times
 * frequency (of 31 and 24 bits, 55 in all) as a sum of two 64-bit numbers, reduced to a part of a turn by a 2 / pi of two
 * more, so that far positions lose nothing before that part becomes fp32.
 *
 * Bound by HBM for prompts: 6300 tokens of 48 heads of 128, 241 MB, 49 us, 4.9 TB/s (a copy of 1 GiB 4.8), by a launch and one
 * chain of loads for few tokens: one token 4.2 us in a graph, 64 of 80 heads 5.3.
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_serve_device.h"

namespace wsr_serve {

constexpr int PT = 256;                       /* threads */
/* Waves of a call, at most, where a token has steps enough: 1801 tokens of 80 heads 25.2 us, with 2048 waves 28, with 12288 28;
   6300 tokens of 48 heads 50, one step a wave (75600 waves) 86. */
constexpr int WAVES = 6144;

/* Over the L lanes of a head. */
template <int L>
__device__ __forceinline__ float head_sum(float v) {
    if constexpr (L == 32) v = wsr::xchg_add<1>(v);
    if constexpr (L >= 16) v = wsr::xchg_add<2>(v);
    return wsr::xchg_add<5>(wsr::xchg_add<4>(wsr::xchg_add<3>(v)));
}

/* Sine and cosine of an angle: whole quarter turns and a rest of at most pi / 4 in 64 bits, of which the series up to x^9 and
   x^8 leave 2^-29 and 2^-25 (0.1 to 0.2 us less than a general function: 1 token of 32 heads on 8 4.2 us, so 4.06).  What the
   product and 2 / pi lose to 64 bits, up to 2^-22 of a quarter at positions of 2^31, is added to the rest, which is then right
   to 2^-53 while there are fewer than 2^45 quarters. */
__device__ __forceinline__ void turn_of(double position, double frequency, float& si, float& co) {
    constexpr double PER = 0.63661977236758134, PER_LOW = -3.9357353350364972e-17;     /* 2 / pi */
    const double angle = position * frequency, low = fma(position, frequency, -angle);
    const double whole = rint(angle * PER), rest = fma(angle, PER, -whole) + fma(low, PER, angle * PER_LOW);
    const float x = (float)rest * 1.5707963267948966f, y = x * x;
    const int n = (int)(whole - 4.0 * floor(whole * 0.25));
    const float s = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), x);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 40320.f, -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const float u = n & 1 ? c : s, v = n & 1 ? s : c;
    si = n & 2 ? -u : u;
    co = (n + 1) & 2 ? -v : v;
}

/* The steps of a token: heads of queries, then of keys, then of values, HW at a time. */
struct Steps {
    int32_t q, k, all;
    int32_t per, chunks;                      /* of a wave, and waves of a token */
};

template <int FMT, int L>
__global__ __launch_bounds__(PT) void k_append(wsr_qkv p, Steps st, int64_t first) {
    constexpr int D = 8 * L, HW = WAVE / L;
    const int64_t w = first + (int64_t)blockIdx.x * (PT / WAVE) + wsr::wave_in_block();
    if (w >= (int64_t)p.n_tokens * st.chunks) return;
    const int tok = (int)(w / st.chunks), from = (int)(w % st.chunks) * st.per, to = min(from + st.per, st.all);
    const int lane = threadIdx.x % WAVE, j = lane % L, sub = lane / L;
    const int half = p.rot_dim / 2;
    const bool turned = 8 * j < p.rot_dim, split = turned && !(p.flags & WSR_QKV_PAIRS);
    const int at0 = split ? 4 * j : 8 * j, at1 = split ? half + 4 * j : 8 * j + 4;

    /* the inputs of a step; those of the next are on their way while one is worked on, the first while the token's place is found */
    struct Run {
        int kind, head, heads;                /* queries, keys, values */
        f4_t a, b;
    };
    auto load = [&](int s) __attribute__((always_inline)) {
        Run r;
        r.kind = s < st.q ? 0 : s < st.q + st.k ? 1 : 2;
        r.head = (r.kind == 0 ? s : r.kind == 1 ? s - st.q : s - st.q - st.k) * HW + sub;
        r.heads = r.kind == 0 ? p.n_heads : p.n_kv_heads;
        const int64_t stride = r.kind == 0 ? p.q_tok_stride : r.kind == 1 ? p.k_tok_stride : p.v_tok_stride;
        const char* x = (const char*)(r.kind == 0 ? p.q : r.kind == 1 ? p.k : p.v) + tok * stride + (int64_t)min(r.head, r.heads - 1) * (4 * D);
        /* read once: 6300 tokens of 48 heads 57.6 us without the hint, so 50.5 */
        r.a = __builtin_nontemporal_load((const f4_t*)(x + 4 * at0)), r.b = __builtin_nontemporal_load((const f4_t*)(x + 4 * at1));
        return r;
    };
    Run next = load(from);

    f4_t freq = f4_t{0.f, 0.f, 0.f, 0.f};
    int pos[4] = {};
    if (turned) {
        freq = *(const wsr_step::f4_any_t*)(p.freqs + 4 * j);
        if (p.positions)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int axis = p.axis_of ? min(max(p.axis_of[4 * j + i], 0), p.n_axes - 1) : 0;
                pos[i] = ((const int32_t*)((const char*)p.positions + axis * p.pos_axis_stride))[tok];
            }
    }

    const Belongs of = seq_of(p.starts, p.n_seqs, tok);
    if (of.seq < 0) return;
    const int64_t place = (int64_t)max(p.lens[of.seq], 0) - min(of.end, p.n_tokens) + tok;
    int page = 0, slot = 0;
    const bool stored = p.k && p.n_kv_heads > 0 && page_of(p.cache, of.seq, place, page, slot);

    float co[4], si[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        co[i] = 1.f, si[i] = 0.f;
        if (!turned) continue;
        turn_of(p.positions ? (double)pos[i] : (double)place, (double)freq[i], si[i], co[i]);
    }

#pragma unroll 1
    for (int s = from; s < to; ++s) {
        const Run r = next;
        if (s + 1 < to) next = load(s + 1);
        f4_t a = r.a, b = r.b;
        if (r.kind < 2) {
            if (p.flags & WSR_QKV_NORM) {
                if (p.kind == WSR_NORM_LAYER) {
                    const float mean = head_sum<L>(((a[0] + a[1]) + (a[2] + a[3])) + ((b[0] + b[1]) + (b[2] + b[3]))) * (1.f / D);
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] -= mean, b[i] -= mean;
                }
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) sq = fmaf(a[i], a[i], fmaf(b[i], b[i], sq));
                const float f = 1.f / sqrtf(head_sum<L>(sq) * (1.f / D) + p.eps);
                const uint16_t *wp = (const uint16_t*)(r.kind ? p.k_w : p.q_w), *bp = (const uint16_t*)(r.kind ? p.k_b : p.q_b);
                float wa[4] = {1.f, 1.f, 1.f, 1.f}, wb[4] = {1.f, 1.f, 1.f, 1.f}, ba[4] = {}, bb[4] = {};
                auto four = [](const uint16_t* from4, float (&v)[4]) {
                    const u32x2 u = *(const u32x2*)from4;
                    unpack2<FMT>(u.x, v[0], v[1]);
                    unpack2<FMT>(u.y, v[2], v[3]);
                };
                if (wp) four(wp + at0, wa), four(wp + at1, wb);
                if (bp) four(bp + at0, ba), four(bp + at1, bb);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = fmaf(a[i] * f, wa[i], ba[i]), b[i] = fmaf(b[i] * f, wb[i], bb[i]);
            }
            if (split) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float u = a[i];
                    a[i] = u * co[i] - b[i] * si[i];
                    b[i] = b[i] * co[i] + u * si[i];
                }
            } else if (turned) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float u = a[2 * i], v = b[2 * i];
                    a[2 * i] = u * co[i] - a[2 * i + 1] * si[i];
                    a[2 * i + 1] = a[2 * i + 1] * co[i] + u * si[i];
                    b[2 * i] = v * co[2 + i] - b[2 * i + 1] * si[2 + i];
                    b[2 * i + 1] = b[2 * i + 1] * co[2 + i] + v * si[2 + i];
                }
            }
        }
        if (r.head >= r.heads || (r.kind && !stored)) continue;
        char* row;
        if (r.kind == 0) row = (char*)p.q_out + tok * p.q_out_tok_stride + r.head * p.q_out_head_stride;
        else row = (char*)(r.kind == 1 ? p.cache.k : p.cache.v) + page * p.cache.page_stride + slot * p.cache.tok_stride + r.head * p.cache.head_stride;
        *(u32x2*)(row + 2 * at0) = u32x2{pack2<FMT>(a[0], a[1]), pack2<FMT>(a[2], a[3])};
        *(u32x2*)(row + 2 * at1) = u32x2{pack2<FMT>(b[0], b[1]), pack2<FMT>(b[2], b[3])};
    }
}

template <int FMT, int L>
static hipError_t launch_dim(const wsr_qkv& p, hipStream_t s) {
    constexpr int HW = WAVE / L;
    const bool cached = p.k && p.n_kv_heads > 0;
    Steps st;
    st.q = p.q ? (p.n_heads + HW - 1) / HW : 0;
    st.k = cached ? (p.n_kv_heads + HW - 1) / HW : 0;
    st.all = st.q + 2 * st.k;
    st.chunks = (int32_t)std::min<int64_t>(st.all, (WAVES + p.n_tokens - 1) / p.n_tokens);
    st.per = (st.all + st.chunks - 1) / st.chunks;
    st.chunks = (st.all + st.per - 1) / st.per;
    const int64_t waves = (int64_t)p.n_tokens * st.chunks, held = most_blocks(PT) * (PT / WAVE);
    for (int64_t first = 0; first < waves; first += held) {
        const int64_t n = (std::min(waves - first, held) + PT / WAVE - 1) / (PT / WAVE);
        hipLaunchKernelGGL((k_append<FMT, L>), dim3((unsigned)n), dim3(PT), 0, s, p, st, first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int FMT>
static hipError_t launch_fmt(const wsr_qkv& p, hipStream_t s) {
    return p.head_dim == 64 ? launch_dim<FMT, 8>(p, s) : p.head_dim == 128 ? launch_dim<FMT, 16>(p, s) : launch_dim<FMT, 32>(p, s);
}

hipError_t launch_append(const wsr_qkv& p, hipStream_t s) {
    return p.fmt == WSR_F16 ? launch_fmt<WSR_F16>(p, s) : launch_fmt<WSR_BF16>(p, s);
}

}  // namespace wsr_serve
