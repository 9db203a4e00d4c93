/*
 * wsr_norm.hip - norms after and before a block, fused with its gate and the residual scale.
 *
 *   v = post(y),  h' = s h + g v,  x = pre(h'):  each row is read once, held in registers through
 *   both norms and written once (14 bytes per element with h' and x), so the kernel is bound by HBM
 *   for prompts (4099 x 8192 layer norms, 537 MB, 97 us, 5.5 TB/s; a copy of 1 GiB reaches 4.8) and by one row's
 *   latency (loads, two or four workgroup sums, stores) for few tokens (one of 4096 3.0 us).
 */
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "wsr_step_device.h"

namespace wsr_step {

typedef const __attribute__((address_space(1))) f4_t g_cf4;
typedef __attribute__((address_space(1))) f4_t g_f4;
typedef const __attribute__((address_space(1))) u32x4 g_cu4;
typedef __attribute__((address_space(1))) u32x4 g_u4;

/* Whether the weights are loaded at the start: with four pieces per thread there are no registers for them. */
template <int NC>
constexpr bool early() { return NC < 4; }

/* u <- (u - mean) / sqrt(var + eps) * w + b over the row's d elements (RMS: mean = 0); w and b where given. */
template <int FMT, int KIND, int WAVES, int NC>
__device__ __forceinline__ void norm_row(float (&u)[NC][8], const u32x4 (&w)[NC], const u32x4 (&b)[NC], const void* wp,
                                         const void* bp, int d, float eps, float (&s0)[WAVES], float (&s1)[WAVES]) {
    const float inv_d = 1.f / (float)d;
    if constexpr (KIND == WSR_NORM_LAYER) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += u[c][j];
        const float mean = block_sum<WAVES>(sum, s0) * inv_d;
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if ((int)(threadIdx.x + c * WAVES * WAVE) * 8 < d)
#pragma unroll
                for (int j = 0; j < 8; ++j) u[c][j] -= mean;
    }
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) sq = fmaf(u[c][j], u[c][j], sq);
    const float r = 1.f / sqrtf(block_sum<WAVES>(sq, s1) * inv_d + eps);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= d) continue;
        float wv[8], bv[8];
        if (wp) unpack8<FMT>(early<NC>() ? w[c] : ((g_cu4*)wp)[i], wv);
        if (bp) unpack8<FMT>(early<NC>() ? b[c] : ((g_cu4*)bp)[i], bv);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[c][j] *= r;
            if (wp) u[c][j] *= wv[j];
            if (bp) u[c][j] += bv[j];
        }
    }
}

/* One workgroup per token; thread i holds elements 8 i .. 8 i + 7 of each run of 8 * threads.  All of the row's
   inputs are loaded at the start (with the gate and the weights loaded where they are used, 4099 x 8192 layer
   norms took 107 us, so 101; one token of 4096 3.43 and 3.30).  STREAM: h' is stored past the caches. */
template <int FMT, int KIND, int WAVES, int NC, bool STREAM>
__global__ __launch_bounds__(WAVES * WAVE) void k_block_norm(wsr_block p) {
    __shared__ float red[4][WAVES];
    const int64_t t = blockIdx.x;
    const int d = (int)p.d;
    float u[NC][8], h[NC][8];
    u32x4 gate[NC], w0[NC], b0[NC], w1[NC], b1[NC];
    const char* yr = (const char*)p.y + t * p.y_tok_stride;
    const char* hr = (const char*)p.h + t * p.h_tok_stride;
    const char* gr = (const char*)p.gate + t * p.gate_tok_stride;
    const bool post = p.y && (p.flags & WSR_BLOCK_POST);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int i = threadIdx.x + c * WAVES * WAVE;
        const bool in = i * 8 < d;
        f4_t a = {0, 0, 0, 0}, b = a, e = a, f = a;
        gate[c] = w0[c] = b0[c] = w1[c] = b1[c] = wsr::zero4();
        if (in) {
            if (p.y) a = ((g_cf4*)yr)[2 * i], b = ((g_cf4*)yr)[2 * i + 1];
            if (p.h) e = ((g_cf4*)hr)[2 * i], f = ((g_cf4*)hr)[2 * i + 1];
            if (p.gate) gate[c] = ((g_cu4*)gr)[i];
            if constexpr (early<NC>()) {
                if (post && p.post_w) w0[c] = ((g_cu4*)p.post_w)[i];
                if (post && p.post_b) b0[c] = ((g_cu4*)p.post_b)[i];
                if (p.x && p.pre_w) w1[c] = ((g_cu4*)p.pre_w)[i];
                if (p.x && p.pre_b) b1[c] = ((g_cu4*)p.pre_b)[i];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) u[c][j] = a[j], u[c][4 + j] = b[j], h[c][j] = e[j], h[c][4 + j] = f[j];
    }
    if (post) norm_row<FMT, KIND, WAVES, NC>(u, w0, b0, p.post_w, p.post_b, d, p.eps, red[0], red[1]);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= d) continue;
        if (p.gate) {
            float g[8];
            unpack8<FMT>(gate[c], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[c][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) u[c][j] = p.h ? fmaf(p.res_scale, h[c][j], u[c][j]) : u[c][j];
        if (p.h_out) {
            g_f4* o = (g_f4*)((char*)p.h_out + t * p.h_out_tok_stride) + 2 * i;
            const f4_t a = {u[c][0], u[c][1], u[c][2], u[c][3]}, b = {u[c][4], u[c][5], u[c][6], u[c][7]};
            if constexpr (STREAM) __builtin_nontemporal_store(a, o), __builtin_nontemporal_store(b, o + 1);
            else o[0] = a, o[1] = b;
        }
    }
    if (!p.x) return;
    norm_row<FMT, KIND, WAVES, NC>(u, w1, b1, p.pre_w, p.pre_b, d, p.eps, red[2], red[3]);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= d) continue;
        ((g_u4*)((char*)p.x + t * p.x_tok_stride))[i] =
            u32x4{pack2<FMT>(u[c][0], u[c][1]), pack2<FMT>(u[c][2], u[c][3]), pack2<FMT>(u[c][4], u[c][5]),
                  pack2<FMT>(u[c][6], u[c][7])};
    }
}

/* As many threads as the row has pieces, up to eight waves: with sixteen the sums take longer than the second pieces
   (rms of 8192 elements, one piece each and two: 1 token 4.8 us, so 4.4; 64 tokens 5.3 and 4.9, 512 13.3 and 12.2;
   4104 elements, 1 token 4.1 and 3.8; 4099 x 8192 layer norms 88.6 and 86.5).  A residual stream larger than the chip's second-level caches is gone from them before it is read
   again, so it is stored past them (8193 x 4096 86.8 us, so 84.8; 8193 x 1160 29.4 and 26.1). */
constexpr int64_t STREAM_FROM = 32 << 20;
template <int FMT, int KIND, int W, int NC>
static hipError_t launch_waves(wsr_block p, hipStream_t s) {
    const bool stream = p.n_tokens * p.d * 4 >= STREAM_FROM;
    /* of its rows as many as a launch holds, then the next */
    auto ahead = [](auto*& at, int64_t bytes) {
        if (at) at = (std::remove_reference_t<decltype(at)>)((const char*)at + bytes);
    };
    for (int64_t left = p.n_tokens, n; left > 0; left -= n) {
        n = std::min(left, most_blocks(W * WAVE));
        const dim3 grid((unsigned)n), threads(W * WAVE);
        if (stream) hipLaunchKernelGGL((k_block_norm<FMT, KIND, W, NC, true>), grid, threads, 0, s, p);
        else hipLaunchKernelGGL((k_block_norm<FMT, KIND, W, NC, false>), grid, threads, 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        ahead(p.y, n * p.y_tok_stride), ahead(p.gate, n * p.gate_tok_stride), ahead(p.h, n * p.h_tok_stride);
        ahead(p.h_out, n * p.h_out_tok_stride), ahead(p.x, n * p.x_tok_stride);
    }
    return hipSuccess;
}
template <int FMT, int KIND>
static hipError_t launch_kind(const wsr_block& p, hipStream_t s) {
    if (p.d <= 512) return launch_waves<FMT, KIND, 1, 1>(p, s);
    if (p.d <= 2048) return launch_waves<FMT, KIND, 4, 1>(p, s);
    if (p.d <= 4096) return launch_waves<FMT, KIND, 8, 1>(p, s);
    if (p.d <= 8192) return launch_waves<FMT, KIND, 8, 2>(p, s);
    if (p.d <= 16384) return launch_waves<FMT, KIND, 16, 2>(p, s);
    return launch_waves<FMT, KIND, 16, 4>(p, s);
}

hipError_t launch_block_norm(const wsr_block& p, hipStream_t s) {
    if (p.fmt == WSR_F16) return p.kind == WSR_NORM_RMS ? launch_kind<WSR_F16, WSR_NORM_RMS>(p, s) : launch_kind<WSR_F16, WSR_NORM_LAYER>(p, s);
    return p.kind == WSR_NORM_RMS ? launch_kind<WSR_BF16, WSR_NORM_RMS>(p, s) : launch_kind<WSR_BF16, WSR_NORM_LAYER>(p, s);
}

}  // namespace wsr_step
