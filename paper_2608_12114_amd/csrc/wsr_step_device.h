/*
 * wsr_step_device.h - device building blocks of the step operators (gfx950, wave64): 16-bit
 * conversions, wave and workgroup reductions, matrix instructions (16 x 16 x 32: wsr_mma.h).
 */
#ifndef WSR_STEP_DEVICE_H
#define WSR_STEP_DEVICE_H

#include "wsr_mma.h"
#include "wsr_step_internal.h"

namespace wsr_step {

using wsr::b8_t;
using wsr::f4_t;
using wsr::h8_t;
using wsr::mma16;
using wsr::u32x4;
using wsr::WAVE;

typedef float f16v_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s4_t __attribute__((ext_vector_type(4)));

/* 16-byte loads and stores of fp32 rows that are only 4-byte aligned (the hardware takes them) */
typedef f4_t f4_any_t __attribute__((aligned(4)));

template <int FMT>
struct Half;
template <>
struct Half<WSR_F16> { typedef _Float16 t; typedef wsr::h2_t t2; };
template <>
struct Half<WSR_BF16> { typedef __bf16 t; typedef wsr::b2_t t2; };

/* The two 16-bit values of a word, low half first. */
template <int FMT>
__device__ __forceinline__ void unpack2(uint32_t v, float& a, float& b) {
    if constexpr (FMT == WSR_BF16) {
        a = __uint_as_float(v << 16);
        b = __uint_as_float(v & 0xffff0000u);
    } else {
        const wsr::h2_t h = __builtin_bit_cast(wsr::h2_t, v);
        a = (float)h.x;
        b = (float)h.y;
    }
}

/* Two values rounded to nearest even and packed. */
template <int FMT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    typename Half<FMT>::t2 v;
    v.x = (typename Half<FMT>::t)a;
    v.y = (typename Half<FMT>::t)b;
    return __builtin_bit_cast(uint32_t, v);
}

template <int FMT>
__device__ __forceinline__ float unpack1(uint16_t v) {
    float a, b;
    unpack2<FMT>(v, a, b);
    return a;
}

template <int FMT>
__device__ __forceinline__ void unpack8(u32x4 w, float (&v)[8]) {
    unpack2<FMT>(w.x, v[0], v[1]);
    unpack2<FMT>(w.y, v[2], v[3]);
    unpack2<FMT>(w.z, v[4], v[5]);
    unpack2<FMT>(w.w, v[6], v[7]);
}

/* Sum over a workgroup of WAVES waves, the same bits in every thread: a wave's tree, then the waves in
   order.  `slot` is a piece of LDS that no other reduction of the kernel uses. */
template <int WAVES>
__device__ __forceinline__ float block_sum(float v, float (&slot)[WAVES]) {
    v = wsr::wave_sum(v);
    if constexpr (WAVES == 1) return v;
    if ((threadIdx.x & (WAVE - 1)) == 0) slot[threadIdx.x / WAVE] = v;
    __syncthreads();
    float s = slot[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) s += slot[i];
    return s;
}

/* Until at most N of the wave's loads (those into LDS among them) are outstanding. */
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

/* Until all of the wave's stores and atomics have arrived (vmcnt counts them beside the loads): those at agent scope, where
   every XCD sees them. */
__device__ __forceinline__ void wait_stores() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

/* v combined with its partner lane's v, by the levels of wsr::xchg_add: lane swaps for levels 0 and 1 (halves,
   then 16-lane rows), moves inside a 16-lane row for levels 2 to 5.  OP must not depend on the order of its
   operands; applied level by level it leaves the same bits in all lanes. */
template <int LEVEL>
__device__ __forceinline__ void partners(uint32_t v, uint32_t& a, uint32_t& b) {
    if constexpr (LEVEL == 0) {
        const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        a = s[0], b = s[1];
    } else if constexpr (LEVEL == 1) {
        const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        a = s[0], b = s[1];
    } else {
        constexpr int CTRL = LEVEL == 2 ? wsr::DPP_MIRROR : LEVEL == 3 ? wsr::DPP_HALF_MIRROR : LEVEL == 4 ? wsr::DPP_XOR2 : wsr::DPP_XOR1;
        a = v;
        b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
    }
}
template <int LEVEL>
__device__ __forceinline__ float xchg_max(float v) {
    uint32_t a, b;
    partners<LEVEL>(__float_as_uint(v), a, b);
    return fmaxf(__uint_as_float(a), __uint_as_float(b));
}
template <int LEVEL>
__device__ __forceinline__ int xchg_min(int v) {
    uint32_t a, b;
    partners<LEVEL>((uint32_t)v, a, b);
    return min((int)a, (int)b);
}

/* Over a 16-lane row. */
__device__ __forceinline__ float row_max(float v) { return xchg_max<5>(xchg_max<4>(xchg_max<3>(xchg_max<2>(v)))); }
__device__ __forceinline__ int row_min(int v) { return xchg_min<5>(xchg_min<4>(xchg_min<3>(xchg_min<2>(v)))); }
__device__ __forceinline__ float row_sum(float v) {
    return wsr::xchg_add<5>(wsr::xchg_add<4>(wsr::xchg_add<3>(wsr::xchg_add<2>(v))));
}
/* Over a wave. */
__device__ __forceinline__ float wave_max(float v) { return row_max(xchg_max<1>(xchg_max<0>(v))); }
__device__ __forceinline__ int wave_min(int v) { return row_min(xchg_min<1>(xchg_min<0>(v))); }

/* D = A B + C on 32 x 32 x 16: lane l holds row l % 32 of A and column l % 32 of B, elements
   8 (l / 32) .. + 7 of their 16; D's column l % 32, register i row 8 (i / 4) + 4 (l / 32) + i % 4. */
template <int FMT>
__device__ __forceinline__ f16v_t mma_32x32x16(u32x4 a, u32x4 b, f16v_t c) {
    if constexpr (FMT == WSR_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8_t, a), __builtin_bit_cast(b8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, a), __builtin_bit_cast(h8_t, b), c, 0, 0, 0);
}

}  // namespace wsr_step

#endif
