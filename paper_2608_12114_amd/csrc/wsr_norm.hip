/*
 * wsr_norm.hip - norms after and before a block, fused with its gate and the residual scale.
 *
 *   v = post(y),  h' = s h + g v,  x = pre(h'):  each row is read once, held in registers through
 *   both norms and written once (14 bytes per element with h' and x), so the kernel is bound by HBM
 *   for prompts and by one row's latency (loads, two or four workgroup sums, stores) for few tokens.
 */
#include <hip/hip_runtime.h>

#include "wsr_step_device.h"

namespace wsr_step {

typedef const __attribute__((address_space(1))) f4_t g_cf4;
typedef __attribute__((address_space(1))) f4_t g_f4;
typedef const __attribute__((address_space(1))) u32x4 g_cu4;
typedef __attribute__((address_space(1))) u32x4 g_u4;

/* u <- (u - mean) / sqrt(var + eps) * w + b over the row's d elements (RMS: mean = 0). */
template <int FMT, int KIND, int WAVES, int NC>
__device__ __forceinline__ void norm_row(float (&u)[NC][8], const void* w, const void* b, int64_t d, float eps,
                                         float (&s0)[WAVES], float (&s1)[WAVES]) {
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
            if ((int64_t)(threadIdx.x + c * WAVES * WAVE) * 8 < d)
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
        const int64_t i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= d) continue;
        float wv[8], bv[8];
        if (w) unpack8<FMT>(((g_cu4*)w)[i], wv);
        if (b) unpack8<FMT>(((g_cu4*)b)[i], bv);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u[c][j] *= r;
            if (w) u[c][j] *= wv[j];
            if (b) u[c][j] += bv[j];
        }
    }
}

/* One workgroup per token; thread i holds elements 8 i .. 8 i + 7 of each run of 8 * threads. */
template <int FMT, int KIND, int WAVES, int NC>
__global__ __launch_bounds__(WAVES * WAVE) void k_block_norm(wsr_block p) {
    __shared__ float red[4][WAVES];
    const int64_t t = blockIdx.x;
    float u[NC][8], h[NC][8];
    const char* yr = (const char*)p.y + t * p.y_tok_stride;
    const char* hr = (const char*)p.h + t * p.h_tok_stride;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int64_t i = threadIdx.x + c * WAVES * WAVE;
        const bool in = i * 8 < p.d;
        f4_t a = {0, 0, 0, 0}, b = a, e = a, f = a;
        if (in && p.y) a = ((g_cf4*)yr)[2 * i], b = ((g_cf4*)yr)[2 * i + 1];
        if (in && p.h) e = ((g_cf4*)hr)[2 * i], f = ((g_cf4*)hr)[2 * i + 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) u[c][j] = a[j], u[c][4 + j] = b[j], h[c][j] = e[j], h[c][4 + j] = f[j];
    }
    if (p.y && (p.flags & WSR_BLOCK_POST))
        norm_row<FMT, KIND, WAVES, NC>(u, p.post_w, p.post_b, p.d, p.eps, red[0], red[1]);
    const char* gr = (const char*)p.gate + t * p.gate_tok_stride;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int64_t i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= p.d) continue;
        if (p.gate) {
            float g[8];
            unpack8<FMT>(((g_cu4*)gr)[i], g);
#pragma unroll
            for (int j = 0; j < 8; ++j) u[c][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) u[c][j] = p.h ? fmaf(p.res_scale, h[c][j], u[c][j]) : u[c][j];
        if (p.h_out) {
            g_f4* o = (g_f4*)((char*)p.h_out + t * p.h_out_tok_stride);
            o[2 * i] = f4_t{u[c][0], u[c][1], u[c][2], u[c][3]};
            o[2 * i + 1] = f4_t{u[c][4], u[c][5], u[c][6], u[c][7]};
        }
    }
    if (!p.x) return;
    norm_row<FMT, KIND, WAVES, NC>(u, p.pre_w, p.pre_b, p.d, p.eps, red[2], red[3]);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int64_t i = threadIdx.x + c * WAVES * WAVE;
        if (i * 8 >= p.d) continue;
        ((g_u4*)((char*)p.x + t * p.x_tok_stride))[i] =
            u32x4{pack2<FMT>(u[c][0], u[c][1]), pack2<FMT>(u[c][2], u[c][3]), pack2<FMT>(u[c][4], u[c][5]),
                  pack2<FMT>(u[c][6], u[c][7])};
    }
}

template <int FMT, int KIND>
static void launch_kind(const wsr_block& p, hipStream_t s) {
#define WSR_NORM(W, NC) \
    hipLaunchKernelGGL((k_block_norm<FMT, KIND, W, NC>), dim3((unsigned)p.n_tokens), dim3(W * WAVE), 0, s, p)
    if (p.d <= 512) WSR_NORM(1, 1);
    else if (p.d <= 2048) WSR_NORM(4, 1);
    else if (p.d <= 4096) WSR_NORM(8, 1);
    else if (p.d <= 8192) WSR_NORM(16, 1);
    else if (p.d <= 16384) WSR_NORM(16, 2);
    else WSR_NORM(16, 4);
#undef WSR_NORM
}

hipError_t launch_block_norm(const wsr_block& p, hipStream_t s) {
    if (p.fmt == WSR_F16) {
        if (p.kind == WSR_NORM_RMS) launch_kind<WSR_F16, WSR_NORM_RMS>(p, s);
        else launch_kind<WSR_F16, WSR_NORM_LAYER>(p, s);
    } else {
        if (p.kind == WSR_NORM_RMS) launch_kind<WSR_BF16, WSR_NORM_RMS>(p, s);
        else launch_kind<WSR_BF16, WSR_NORM_LAYER>(p, s);
    }
    return hipGetLastError();
}

}  // namespace wsr_step
