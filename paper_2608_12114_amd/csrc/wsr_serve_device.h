/*
 * wsr_serve_device.h - device building blocks of the serving operators (gfx950, wave64): tokens and their sequences,
 * places and their pages.
 */
#ifndef WSR_SERVE_DEVICE_H
#define WSR_SERVE_DEVICE_H

#include "wsr_serve_internal.h"
#include "wsr_step_device.h"

namespace wsr_serve {

using wsr::f4_t;
using wsr::u32x4;
using wsr::WAVE;
using wsr_step::most_blocks;
using wsr_step::pack2;
using wsr_step::u32x2;
using wsr_step::unpack2;
using wsr_step::unpack8;

constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.4426950408889634f;

/* Lanes of a wave hand each other values through LDS: what was stored is there for the loads that follow, what was loaded has
   been read before the stores that follow.  No instruction, as a wave's LDS operations are done in order; the compiler may not
   move them across. */
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }

/* The sequence that row `tok` belongs to (-1: none) and the row behind its last: the last sequence that starts at or before
   it, by a search of 64 samples at a time (one load's latency below 64 sequences, two below 4096).  By whole waves, tok
   uniform. */
struct Belongs {
    int seq, end;
};
__device__ __forceinline__ Belongs seq_of(const int32_t* starts, int n_seqs, int tok) {
    if (!starts) return Belongs{tok < n_seqs ? tok : -1, tok + 1};
    const int lane = threadIdx.x % WAVE;
    int lo = 0, n = n_seqs + 1;               /* how many start at or before tok: lo to lo + n */
    int first = 0, end = 0;                   /* starts[lo - 1] and, where it was among the samples, starts[lo] */
    bool ended = false;
    while (n > 0) {
        const int step = (n + WAVE - 1) / WAVE, at = lane * step, all = (n + step - 1) / step;
        const int v = at < n ? starts[lo + at] : 0;
        const int c = __builtin_popcountll(__ballot(at < n && v <= tok));
        if (c == 0) break;
        first = __builtin_amdgcn_readlane(v, c - 1);
        ended = step == 1 && c < all;
        if (ended) end = __builtin_amdgcn_readlane(v, c);
        lo += (c - 1) * step + 1;
        n = min(step - 1, n - (c - 1) * step - 1);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    if (lo < 1 || lo > n_seqs) return Belongs{-1, 0};
    if (!ended) end = starts[lo];
    return Belongs{first <= tok && tok < end ? lo - 1 : -1, end};
}

/* The page of a place, and whether it is one. */
__device__ __forceinline__ bool page_of(const wsr_pages& c, int seq, int64_t place, int& page, int& slot) {
    if (place < 0 || place >= (int64_t)c.max_pages * c.page_size) return false;
    const uint32_t at = (uint32_t)place / (uint32_t)c.page_size;
    slot = (int)((uint32_t)place - at * (uint32_t)c.page_size);
    page = ((const int32_t*)((const char*)c.table + seq * c.table_stride))[at];
    return (uint32_t)page < (uint32_t)c.n_pages;
}

}  // namespace wsr_serve

#endif
