/*
 * wsr_attend.h - a workgroup's attention over blocks of keys that lie in its LDS: products, running maximum and sum, and the
 * join of the waves' results, whatever memory the blocks come from.
 */
#ifndef WSR_ATTEND_H
#define WSR_ATTEND_H

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int AT = 256, AW = AT / WAVE;
constexpr float A_NEG_INF = -__builtin_inff();
constexpr float A_LOG2E = 1.4426950408889634f;

typedef __attribute__((address_space(3))) u32x4 l_u32x4;
typedef __attribute__((address_space(3))) char l_char;
typedef __attribute__((address_space(3))) s4_t l_s4;

/* The running maximum is only moved when a row's scores pass it by 2^LAZY: until then its probabilities are
   taken against the old one (at most 2^LAZY, exact after the division by their sum), and the sums and
   outputs need no rescaling. */
constexpr float LAZY = 8.f;

/* log of a row's sum l against its maximum m: -inf where it saw no key, and NaN, like its outputs, where a score was NaN,
   which leaves no trace in the maximum. */
__device__ __forceinline__ float lse_of(float m, float l, float scale) { return l == 0.f ? A_NEG_INF : m * scale + logf(l); }

/* A workgroup's place: RW waves side by side over rows (32 each), KW = 4 / RW groups of them over
   alternate blocks of KT keys. */
template <int FMT, int D, int RW>
struct AttendBlocks {
    static constexpr int KW = AW / RW, KT = KW == 1 && D < 256 ? 64 : 32, TILES = KT / 32;
    static constexpr int PIECES = D / 8;                        /* 16-byte pieces of a key */
    static constexpr int ROW = 2 * D;                           /* bytes of a key */
    static constexpr int HALF = KT * PIECES;                    /* pieces of a block of keys (and of values) */
    static constexpr int BUFFER = 2 * HALF * 16;                /* bytes of one of a group's two buffers */
    static constexpr int LOADS = HALF / WAVE / RW;              /* of 64 pieces, per wave and plane */
    static constexpr int DT = D / 32, KS = D / 16;
    static constexpr int LDS = KW * 2 * 2 * HALF;               /* pieces of the workgroup */

    u32x4 q[KS];
    f16v_t o[DT];
    float m, l;                                                 /* the maximum that probabilities are taken against; this half's sum */
    uint32_t ka[KS], va[DT];                                    /* a lane's places in LDS */

    /* Piece x of a key lies at x ^ swz: the 16 keys of a read of keys, and the four keys times four pieces of a
       transposing read of values, lie on the 64 banks once each (two keys of 64 share a round of banks). */
    static __device__ __forceinline__ int kswz(int key) { return D >= 128 ? key & 15 : key >> 1 & 7; }
    static __device__ __forceinline__ int vswz(int key) {
        return D >= 128 ? (key & 3) << 2 | (key >> 2 & 1) : (key >> 1 & 1) << 2 | (key >> 2 & 1);
    }

    /* Places relative to the first group's first buffer, `base` bytes on for the wave's own group. */
    __device__ __forceinline__ void init(uint32_t base, int lane) {
        const int col = lane % 32, h = lane / 32, r = lane % 16 / 4, c = 2 * (col / 16) + lane % 4 / 2;
#pragma unroll
        for (int k = 0; k < KS; ++k) ka[k] = base + col * ROW + ((2 * k + h) ^ kswz(col)) * 16;
#pragma unroll
        for (int i = 0; i < DT; ++i)
            va[i] = base + HALF * 16 + (4 * h + r) * ROW + ((4 * i + c) ^ vswz(4 * h + r)) * 16 + lane % 2 * 8;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
        m = A_NEG_INF, l = 0.f;
    }

    /* One block of keys in buffer `buf` (of the first group): `left` keys of it are visible to this lane's row, where the bits
       of `there` are set. */
    __device__ __forceinline__ void step(const l_char* buf, int left, bool masked, float c, int lane, uint64_t there = ~0ull) {
        const int h = lane / 32;
        f16v_t s[TILES];
        u32x4 kf[TILES][KS];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int k = 0; k < KS; ++k)
                kf[t][k] = *(const l_u32x4*)(buf + ka[k] + 32 * t * ROW);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) s[t][j] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) s[t] = mma_32x32x16<FMT>(kf[t][k], q[k], s[t]);
        }
        /* AHEAD reads before the products, then one read after each */
        constexpr int AHEAD = KS < 6 ? KS : 6;
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < TILES * KS - AHEAD; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
        /* values of 16 keys at a time, the next 16 in flight */
        u32x4 vf[2][DT];
        auto values = [&](u32x4 (&f)[DT], int t, int k) {
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32x2 w = __builtin_bit_cast(
                        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((l_s4*)(buf + va[i] + (32 * t + 16 * k + 8 * e) * ROW)));
                    f[i][2 * e] = w.x, f[i][2 * e + 1] = w.y;
                }
        };
        __builtin_amdgcn_sched_barrier(0);
        values(vf[0], 0, 0);
        if (masked) {
            asm volatile("");                                   /* a branch: without it every block pays for the selects */
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                {
                    const int key = 32 * t + 8 * (j / 4) + 4 * h + j % 4;
                    if (key >= left || !(there >> key & 1)) s[t][j] = A_NEG_INF;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int j = 0; j < 16; ++j) top = fmaxf(top, s[t][j]);
        top = xchg_max<0>(top);
        /* (top - m) c > LAZY, true too where m is -inf and top is not */
        if (__ballot((top - m) * c > LAZY)) {
            const float next = fmaxf(m, top), f = next == A_NEG_INF ? 1.f : __builtin_amdgcn_exp2f((m - next) * c);
            l *= f;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= f;
            m = next;
        }
        const float base = m == A_NEG_INF ? 0.f : m * c;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                s[t][j] = __builtin_amdgcn_exp2f(fmaf(s[t][j], c, -base));
                l += s[t][j];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {                       /* 16 keys */
                if (t + 1 < TILES || k == 0) values(vf[(k + 1) & 1], k == 0 ? t : t + 1, (k + 1) & 1);
                u32x4 pt;
#pragma unroll
                for (int j = 0; j < 4; ++j) pt[j] = pack2<FMT>(s[t][8 * k + 2 * j], s[t][8 * k + 2 * j + 1]);
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = mma_32x32x16<FMT>(vf[k][i], pt, o[i]);
            }
        }
    }

    /* The products take masked keys with a probability of zero, and zero times an infinity or NaN among their values
       would reach rows that do not see them.  Such a row is found by its output (after join()) and summed up again,
       key by key over those it sees, against the maximum it has: nothing is paid for it in the loop (replacing such
       values in LDS there cost 3 to 7 % of every call).  One with a NaN among its scores is NaN throughout and is left
       alone (a NaN in one query's q, 63 tokens behind 4001 keys: summed up again 503 us, so 51, as without; 4 prompts of
       900 behind 8192 6748 and 418, where the check costs 3 of 370 us without any). */
    __device__ __forceinline__ bool broken() const {
        float z = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) z = fmaf(o[i][j], 0.f, z);
        z = wsr::xchg_add<0>(z);
        return z != z;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    }

    /* Adds up the groups' results in LDS; the first group's waves hold the row's maximum, sum (both halves)
       and output afterwards. */
    __device__ __forceinline__ void join(u32x4* lds, float c, int wave, int lane) {
        l = wsr::xchg_add<0>(l);
        if constexpr (KW > 1) {
            float* f = (float*)lds;
            constexpr int PER = WAVE * (16 * DT + 2);           /* floats that a wave leaves */
            static_assert((AW - RW) * PER * 4 <= LDS * 16, "the waves' results fit the key buffers");
            if (wave >= RW) {
                float* w = f + (wave - RW) * PER + lane;
                w[0] = m, w[WAVE] = l;
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[(2 + 16 * i + j) * WAVE] = o[i][j];
            }
            __syncthreads();
            if (wave < RW) {
#pragma unroll
                for (int g = 1; g < KW; ++g) {
                    const float* w = f + ((g - 1) * RW + wave) * PER + lane;
                    const float m2 = w[0], top = fmaxf(m, m2), base = top == A_NEG_INF ? 0.f : top * c;
                    const float a = __builtin_amdgcn_exp2f(m * c - base), b = __builtin_amdgcn_exp2f(m2 * c - base);
                    l = l * a + w[WAVE] * b;
                    m = top;
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[i][j] = o[i][j] * a + w[(2 + 16 * i + j) * WAVE] * b;
                }
            }
        }
    }
};

}  // namespace wsr_step

#endif
