/*
 * wsr_paged_rows.hip - paged attention of many rows: drafts of many heads, and chunks of prompts.
 *
 * A workgroup takes a tile of 64 or 128 rows, 32 to a wave, so that a block of keys and values that is fetched into LDS once
 * serves all of them; wsr_attend.h does the rest.  Blocks alternate between two buffers, one fetched while the other is
 * worked on: a lane knows the place of one key, the places of the pieces that it fetches come from the other lanes, and
 * the pages of the block after it are looked up meanwhile.  Heads of 256 have blocks of 32 keys and one workgroup a CU: 2 chunks
 * of up to 512 tokens behind 4096, 16 heads on 4, 88 us (in tiles of 32 rows, eight times the reads, 173).
 *
 * Chunks of prompts are bound by the matrix cores and the exponentials between their products, as attention behind a prefix
 * is: 2 chunks of up to 512 tokens behind 4096, 32 heads on 8, 39 GFLOP, 72 us with the join (61 without, 640 TFLOP/s).  Drafts
 * by the loads, one block in flight for each workgroup: 24 sequences of 5 with up to 6001 keys, 64 heads on 8, 280 MB, 63 us with
 * the join (54 without, 5.2 TB/s), without the hint that a tile that holds all of a sequence's rows is read once 70.
 */
#include <hip/hip_runtime.h>

#include "wsr_attend.h"
#include "wsr_paged.h"

namespace wsr_serve {

using wsr_step::AT;
using wsr_step::l_char;

typedef __attribute__((address_space(1))) const char g_char;

template <int FMT, int D, int RW, bool ONCE>  /* ONCE: hinted that keys are read once */
struct PagedBlocks : wsr_step::AttendBlocks<FMT, D, RW> {
    typedef wsr_step::AttendBlocks<FMT, D, RW> B;
    using B::HALF, B::KS, B::DT, B::KT, B::KW, B::LOADS, B::PIECES, B::BUFFER, B::q, B::o, B::m, B::kswz, B::vswz, B::step;

    static constexpr int HINT = ONCE ? 2 : 0;                   /* non-temporal */
    int64_t off;                                                /* of the fetched block's key lane % KT */
    int entry, slot;                                            /* and of the next one's */
    uint64_t there;                                             /* the fetched block's keys that are on a page */

    __device__ __forceinline__ void look_up(const wsr_pages& c, const PagedPlan& pl, const int32_t* table, int at, int k1, int lane) {
        const int key = min(at + lane % KT, k1 - 1);
        const int page = (int)((uint64_t)key * pl.magic >> pl.shift);
        slot = key - page * c.page_size;
        entry = table[page];
    }
    /* Block at .. + KT - 1 into a buffer of the group; keys that are not there repeat the first that is, or, where none is,
       `some` readable row. */
    __device__ __forceinline__ void fetch(const wsr_pages& c, const char* kb, const char* vb, const char* some, int at, int k1,
                                          l_char* buf, int rwave, int lane) {
        lane = opaque(lane);
        there = __ballot((uint32_t)entry < (uint32_t)c.n_pages && at + lane % KT < k1);
        off = entry * c.page_stride + slot * c.tok_stride;
        if (!there) {
            off = 0, kb = vb = some;
        } else if (there != ~0ull) {
            const int f = __builtin_ctzll(there);
            const int64_t first = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(off >> 32), f) << 32 |
                                            (uint32_t)__builtin_amdgcn_readlane((int)off, f));
            if (!(there >> lane & 1)) off = first;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int place = (rwave * LOADS + i) * WAVE, key = (place + lane) / PIECES, piece = (place + lane) % PIECES;
            const int64_t from = __shfl((long long)off, key);
            __builtin_amdgcn_global_load_lds((g_char*)(kb + from + 16 * (piece ^ kswz(key))), buf + place * 16, 16, 0, HINT);
            __builtin_amdgcn_global_load_lds((g_char*)(vb + from + 16 * (piece ^ vswz(key))), buf + (HALF + place) * 16, 16, 0, HINT);
        }
    }
    /* Adds key by key those from .. to - 1, where they are there and before lim. */
    __device__ __forceinline__ void again(const wsr_pages& c, const int32_t* table, const char* kb, const char* vb, int from, int to,
                                          int lim, float scale, int lane) {
        const int h = lane / 32;
        const float base = m == NEG_INF ? 0.f : m * scale;
#pragma unroll 1
        for (int key = from; key < to; ++key) {
            const int page = key / c.page_size, at = table[page];
            if ((uint32_t)at >= (uint32_t)c.n_pages) continue;
            const int64_t off1 = at * c.page_stride + (key - page * c.page_size) * c.tok_stride;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const u32x4 w = ((const u32x4*)(kb + off1))[2 * k + h];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float a, b, x, y;
                    unpack2<FMT>(w[j], a, b);
                    unpack2<FMT>(q[k][j], x, y);
                    s = fmaf(a, x, fmaf(b, y, s));
                }
            }
            s = wsr::xchg_add<0>(s);
            const bool see = key < lim;
            const float prob = see ? __builtin_amdgcn_exp2f(fmaf(s, scale, -base)) : 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x2 w = *(const u32x2*)(vb + off1 + (32 * i + 8 * j + 4 * h) * 2);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float a, b;
                        unpack2<FMT>(see ? w[e] : 0u, a, b);
                        o[i][4 * j + 2 * e] = fmaf(prob, a, o[i][4 * j + 2 * e]);
                        o[i][4 * j + 2 * e + 1] = fmaf(prob, b, o[i][4 * j + 2 * e + 1]);
                    }
                }
        }
    }
};

template <int FMT, int D, int RW, bool ONCE>
__global__ __launch_bounds__(AT) __attribute__((amdgpu_waves_per_eu(D == 256 ? 1 : 2))) void k_paged_rows(wsr_paged p, PagedPlan pl) {
    typedef PagedBlocks<FMT, D, RW, ONCE> A;
    __shared__ u32x4 lds_room[A::LDS];
    l_char* lds = (l_char*)lds_room;
    constexpr int R = 32 * RW, STEP = A::KT * A::KW;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), rwave = wave % RW, group = wave / RW, col = lane % 32;
    const int G = p.n_heads / p.n_kv_heads, N = p.n_kv_heads;
    Place place;
    if (!find(p, pl, blockIdx.x, false, place)) return;
    const Seq s = place.s;
    /* key heads side by side: of eight of them each stays on one XCD, whose L2 holds the keys that its tiles share (8
       sequences of 9 tokens 21.4 us with a head's parts side by side, so 20.9) */
    const int parts = place.parts, head = place.at % N, part = place.at / N % parts, tile = place.at / N / parts;
    const int row0 = tile * R, last = min(row0 + R, s.rows) - 1, past = s.len - s.n;
    const int seen = max(past + last / G + 1, 0);
    const int each = ((seen + parts - 1) / parts + STEP - 1) / STEP * STEP;
    const int k0 = (int)min((int64_t)part * each, (int64_t)seen), k1 = seen - k0 > each ? k0 + each : seen;
    const char* kb = (const char*)p.cache.k + head * p.cache.head_stride;
    const char* vb = (const char*)p.cache.v + head * p.cache.head_stride;
    const int32_t* table = (const int32_t*)((const char*)p.cache.table + place.seq * p.cache.table_stride);
    const char* some = (const char*)p.q + s.t0 * p.q_tok_stride + head * G * p.q_head_stride;
    const int lim = past + min(row0 + rwave * 32 + col, last) / G + 1;
    /* of the wave's rows: keys that all see, and that one does */
    const int low = past + min(row0 + rwave * 32, last) / G + 1;
    const int high = row0 + rwave * 32 > last ? 0 : past + min(row0 + rwave * 32 + 31, last) / G + 1;
    const float c = p.scale * LOG2E;

    A a;
    const uint32_t group_at = group * 2 * A::BUFFER;
    a.init(group_at, lane);
    int at = k0 + group * A::KT;
    uint64_t there = 0;
    if (at < k1) {
        a.look_up(p.cache, pl, table, at, k1, lane);
        a.fetch(p.cache, kb, vb, some, at, k1, lds + group_at, rwave, lane);
        a.look_up(p.cache, pl, table, at + STEP, k1, lane);
        there = a.there;
    }
    {
        const int row = min(row0 + rwave * 32 + col, last);
        const char* qr = (const char*)p.q + (s.t0 + row / G) * p.q_tok_stride + (head * G + row % G) * p.q_head_stride;
#pragma unroll
        for (int k = 0; k < A::KS; ++k) a.q[k] = ((const u32x4*)qr)[2 * k + lane / 32];
    }
    /* the two buffers are declared not to alias, so that the compiler does not wait for the loads into one before it reads
       the other */
    auto round = [&](const l_char* __restrict cur, l_char* __restrict next) __attribute__((always_inline)) {
        wsr_step::wait_loads<0>();
        __syncthreads();                                        /* `cur` is there, `next` has been read */
        const uint64_t now = there;
        if (at + STEP < k1) {
            a.fetch(p.cache, kb, vb, some, at + STEP, k1, next + group_at, rwave, lane);
            a.look_up(p.cache, pl, table, at + 2 * STEP, k1, lane);
            there = a.there;
        }
        const int end = min(at + A::KT, k1);
        if (at < min(end, high)) a.step(cur, min(lim, end) - at, min(low, end) < at + A::KT || now != ~0ull, c, lane, now);
        at += STEP;
    };
#pragma unroll 1
    for (int left = (k1 - k0 + STEP - 1) / STEP; left > 0; left -= 2) {
        round(lds, lds + A::BUFFER);
        if (left == 1) break;
        round(lds + A::BUFFER, lds);
    }
    __syncthreads();
    a.join(lds_room, c, wave, lane);
    if (wave >= RW) return;
    /* rows that an infinity or NaN among values they do not see has reached, summed up again; a NaN sum is the row's own */
    const bool mine = a.broken() && a.l == a.l;
    if (__ballot(mine)) {
        if (mine) a.clear();
        a.again(p.cache, table, kb, vb, k0, k1, mine ? lim : 0, c, lane);
    }
    const int row = row0 + rwave * 32 + opaque(lane) % 32, h = lane / 32;
    if (row > last) return;
    const int tok = s.t0 + row / G, qh = head * G + row % G;
    if (parts == 1) {
        const float inv = inverse_of(a.l);
        char* out = (char*)p.out + tok * p.out_tok_stride + qh * p.out_head_stride;
#pragma unroll
        for (int i = 0; i < A::DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(u32x2*)(out + (32 * i + 8 * j + 4 * h) * 2) =
                    u32x2{pack2<FMT>(a.o[i][4 * j] * inv, a.o[i][4 * j + 1] * inv), pack2<FMT>(a.o[i][4 * j + 2] * inv, a.o[i][4 * j + 3] * inv)};
        if (p.lse && h == 0) p.lse[(int64_t)tok * p.n_heads + qh] = lse_of(a.m, a.l, p.scale);
    } else {
        const int to_slot = place.slot + (tile * N + head) * parts + part;
        if ((uint32_t)to_slot >= (uint32_t)pl.slots) return;
        float* w = pl.part + ((int64_t)to_slot * R + row - row0) * (D + 4);
#pragma unroll
        for (int i = 0; i < A::DT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *(f4_t*)(w + 32 * i + 8 * j + 4 * h) = f4_t{a.o[i][4 * j], a.o[i][4 * j + 1], a.o[i][4 * j + 2], a.o[i][4 * j + 3]};
        if (h == 0) w[D] = a.m, w[D + 1] = a.l;
    }
}

template <int FMT, int D>
static hipError_t launch_dim(const wsr_paged& p, const PagedPlan& pl, int rw, bool once, int64_t blocks, hipStream_t s) {
    const dim3 grid((unsigned)blocks), threads(AT);
    if (rw == 4) hipLaunchKernelGGL((k_paged_rows<FMT, D, 4, false>), grid, threads, 0, s, p, pl);
    else if (once) hipLaunchKernelGGL((k_paged_rows<FMT, D, 2, true>), grid, threads, 0, s, p, pl);
    else hipLaunchKernelGGL((k_paged_rows<FMT, D, 2, false>), grid, threads, 0, s, p, pl);
    return hipGetLastError();
}

template <int FMT>
static hipError_t launch_fmt(const wsr_paged& p, const PagedPlan& pl, int rw, bool once, int64_t blocks, hipStream_t s) {
    return p.head_dim == 64    ? launch_dim<FMT, 64>(p, pl, rw, once, blocks, s)
           : p.head_dim == 128 ? launch_dim<FMT, 128>(p, pl, rw, once, blocks, s)
                               : launch_dim<FMT, 256>(p, pl, rw, once, blocks, s);
}

hipError_t launch_paged_rows(const wsr_paged& p, const PagedPlan& pl, int rw, bool once, int64_t blocks, hipStream_t s) {
    return p.fmt == WSR_F16 ? launch_fmt<WSR_F16>(p, pl, rw, once, blocks, s) : launch_fmt<WSR_BF16>(p, pl, rw, once, blocks, s);
}

}  // namespace wsr_serve
