/*
 * wsr_paged.h - how the work of paged attention is cut: units, their parts, and the slots those leave their results in.
 *
 * Items are the parts of all units, sequence after sequence.  Where sequences are few, every wave finds its item by sums over
 * all of them, a lane to each of 64 at a time.  The reads of all workgroups grow with the square of the sequences there (2^20 of
 * them would take minutes), so where they are many one workgroup writes the sums up to each sequence first (k_paged_line) and a
 * wave searches those, 64 ways a step.
 */
#ifndef WSR_PAGED_H
#define WSR_PAGED_H

#include "wsr_serve_device.h"

namespace wsr_serve {

struct Cut {
    float inv, up;                            /* one over the keys of a part; what is added before the number of parts is rounded down */
};
struct Upto {
    int32_t items, slots;                     /* of the sequences before one, LINE_END at most */
};
constexpr int32_t LINE_END = 1 << 30;         /* more than a launch has workgroups */
struct Line {
    Cut cut;
    Upto upto[1];                             /* [n_seqs] */
};

struct PagedPlan {
    int32_t rows;                             /* R, rows of a tile */
    int32_t held;                             /* workgroups that the chip holds at a time */
    int32_t slots;                            /* of parts */
    int32_t whole;                            /* no unit is cut */
    int32_t shift;                            /* division by page_size: (n * magic) >> shift for n < 2^31 */
    uint64_t magic;
    float* part;                              /* [slots][R][head_dim + 4] */
    Line* line;                               /* of many sequences, as k_paged_line leaves it; else null */
};

/* ---- units and their parts -------------------------------------------------------------------------- */

struct Seq {
    int32_t t0, n, len;                       /* first token, tokens, keys */
    int32_t rows, tiles;
};
__device__ __forceinline__ Seq seq_at(const wsr_paged& p, int R, int b) {
    Seq s;
    int next;
    if (p.starts) {
        s.t0 = min(max(p.starts[b], 0), p.n_tokens);
        next = min(max(p.starts[b + 1], s.t0), p.n_tokens);
    } else s.t0 = b, next = b + 1;
    s.n = next - s.t0;
    s.len = (int)min(max((int64_t)p.lens[b], (int64_t)0), p.max_len);
    s.rows = s.n * (p.n_heads / p.n_kv_heads);
    s.tiles = (s.rows + R - 1) / R;
    return s;
}

/* Where units are few against the workgroups that the chip holds, an eighth of them, or half for tiles of more than 32 rows,
   they are cut into as many parts as fill it once, the shorter ones rounded up (7 sequences of up to 65536 keys 257 us in a
   graph, in one and a half rounds 267; 24 of 5 drafts of 8 heads 63, by the other rule 74).  Otherwise parts are half of what
   falls to a workgroup, and units of less than two such stay whole, so that whoever is done early takes another (16 sequences
   of 2000 with 32 key heads 58 us, by the first rule 67; 32 of up to 4096 63, with parts two thirds or four thirds as long 65).
   Parts are meant to have 256 keys or more, of 64 (128) rows 448 (704), since their rows have to be written and read again; as
   their number is rounded up where units are few, and a unit's keys are shared out in whole rounds of its workgroup's blocks,
   the last ones may have a few keys or none (of 257 keys 256 and 1; 32771 are 95 parts, of which 85 have 384, one the rest).
   Sums of lengths are fp32, with every product's rounding written out: all waves of both kernels have to cut alike. */
struct Sums {
    float keys, units;
    __device__ __forceinline__ void add(const Seq& s, int N) {
        const float of = (float)(s.tiles * N);
        units += of, keys = fmaf(of, (float)s.len, keys);
    }
};
__host__ __device__ __forceinline__ float few_units(const PagedPlan& pl) { return (float)pl.held * (pl.rows > 32 ? 0.5f : 0.125f); }
/* Parts of the keys over `share`, where that is enough for one. */
__device__ __forceinline__ Cut cut_by(const PagedPlan& pl, float inv_keys, float share, float up) {
    return Cut{fminf(__builtin_amdgcn_rcpf((float)(192 + 4 * pl.rows)), share * inv_keys), up};
}
/* The cut by sums over all sequences; where units are few, as it is before any tries. */
__device__ __forceinline__ Cut cut_of(const PagedPlan& pl, const Sums& sums) {
    const float inv_keys = __builtin_amdgcn_rcpf(sums.keys), held = (float)pl.held;
    return sums.units <= few_units(pl) ? cut_by(pl, inv_keys, held - sums.units, 0.999f) : cut_by(pl, inv_keys, held * 2.f, 0.f);
}
/* Parts of each of a sequence's units. */
__device__ __forceinline__ int parts_of(const Seq& s, Cut cut) {
    return (int)fminf(fmaxf(floorf(fmaf((float)s.len, cut.inv, cut.up)), 1.f), 2048.f);
}

/* The lanes' sums of themselves and those below: inside 16-lane rows, then the rows' last lanes handed on. */
__device__ __forceinline__ int scan32(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     /* from one lane below, two, four, eight */
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     /* lane 15 of a row to the next, of rows 1 and 3 */
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);     /* lane 31 to rows 2 and 3 */
    return v;
}

struct Place {
    Seq s;
    int seq, at, parts, slot;                 /* at: item of the sequence; slot: of the sequence's first part */
};
/* find() by the sums up to each sequence: the last one that no more than `item` items lie before. */
__device__ __forceinline__ bool find_upto(const wsr_paged& p, const PagedPlan& pl, int item, bool by_seq, Place& o) {
    const int lane = threadIdx.x % WAVE;
    int b = by_seq ? item : 0;
    for (int n = by_seq ? 1 : p.n_seqs; n > 1;) {               /* among b .. b + n - 1, and none lies before b */
        const int step = (n + WAVE - 1) / WAVE, at = lane * step;
        const int c = __builtin_popcountll(__ballot(at < n && pl.line->upto[b + min(at, n - 1)].items <= item));
        b += (c - 1) * step, n = min(step, n - (c - 1) * step);
    }
    auto of = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    b = of(b);
    const Seq s = seq_at(p, pl.rows, b);
    o.s = Seq{of(s.t0), of(s.n), of(s.len), of(s.rows), of(s.tiles)};
    o.seq = b, o.parts = pl.whole ? 1 : of(parts_of(s, pl.line->cut)), o.at = item - of(pl.line->upto[b].items), o.slot = of(pl.line->upto[b].slots);
    return by_seq || (o.at >= 0 && (int64_t)(o.s.tiles * p.n_kv_heads) * o.parts > o.at);
}
/* Item `item` of the call, or (by_seq) the first of sequence `item`: its sequence, how that is cut and where its parts lie.
   False where there is no such item. */
__device__ __forceinline__ bool find(const wsr_paged& p, const PagedPlan& pl, int item, bool by_seq, Place& o) {
    const int lane = threadIdx.x % WAVE, N = p.n_kv_heads;
    /* sequence b of those from lo on, nothing from lo + n on; loads without a branch, so that several are on their way at once */
    auto seq_in = [&](int b, int lo, int n) {
        Seq s = seq_at(p, pl.rows, min(lo + b, p.n_seqs - 1));
        if (b >= n) s.rows = s.tiles = s.n = s.len = 0;
        return s;
    };
    Seq s = seq_in(lane, 0, p.n_seqs);        /* on its way before the branch: one sequence of 500 8.2 us, behind it 8.4 */
    if (pl.line) return find_upto(p, pl, item, by_seq, o);
    Cut cut{1.f, 0.f};
    if (!pl.whole) {
        Sums sums{0.f, 0.f};
        sums.add(s, N);
#pragma unroll 4
        for (int b = WAVE; b < p.n_seqs; b += WAVE) sums.add(seq_in(b + lane, 0, p.n_seqs), N);
        sums.keys = wsr::wave_sum(sums.keys), sums.units = wsr::wave_sum(sums.units);
        cut = cut_of(pl, sums);
        if (sums.units <= few_units(pl) && p.n_seqs >= 8 && p.n_seqs <= WAVE) {
            /* a sequence's last part is rounded up by half of one, not by one: in four tries the shortest parts that the
               chip holds at once (24 sequences of 5 drafts 66.7 us, so 63.3; where sequences are fewer, nothing) */
            const float inv_keys = __builtin_amdgcn_rcpf(sums.keys);
            float share = (float)pl.held - sums.units, by = sums.units * 0.5f;
#pragma unroll 1
            for (int i = 0; i < 4; ++i, by *= 0.5f) {
                const Cut next = cut_by(pl, inv_keys, share + by, 0.999f);
                const int all = __builtin_amdgcn_readlane(scan32(s.tiles * N * parts_of(s, next)), WAVE - 1);
                if (next.inv == cut.inv) break;
                if (all <= pl.held) cut = next, share += by;
            }
        }
    }
    int lo = 0, n = p.n_seqs;                 /* the sequences left, and items and slots of those before them */
    int items = 0, slots = 0;
    while (true) {                            /* to a 64th of them at a time */
        const int per = (n + WAVE - 1) / WAVE;
        int parts = 1, all = 0, cuts = 0;
        auto count = [&]() __attribute__((always_inline)) {
            if (!pl.whole) parts = parts_of(s, cut);
            const int mine = s.tiles * N * parts;
            all += mine, cuts += parts > 1 ? mine : 0;
        };
        if (per == 1) {
            if (p.n_seqs > WAVE) s = seq_in(lane, lo, n);
            count();
        } else {
            const int end = min(lane * per + per, n);
#pragma unroll 4
            for (int i = 0; i < per; ++i) s = seq_in(lane * per + i, lo, end), count();
        }
        const int to = scan32(all), cuts_to = pl.whole ? 0 : scan32(cuts);
        const uint64_t here = __ballot(by_seq ? (uint32_t)(item - lo - lane * per) < (uint32_t)per : items + to > item);
        if (!here) return false;
        const int w = __builtin_ctzll(here);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, w); };
        items += of(to) - of(all), slots += of(cuts_to) - of(cuts);
        if (per == 1) {
            o.s = Seq{of(s.t0), of(s.n), of(s.len), of(s.rows), of(s.tiles)};
            o.seq = lo + w, o.parts = of(parts), o.at = item - items, o.slot = slots;
            /* starts that decrease may count more than 32 bits hold */
            return by_seq || (o.at >= 0 && (int64_t)(o.s.tiles * N) * o.parts > o.at);
        }
        lo += w * per, n = min(per, n - w * per);
    }
}

/* log of a row's sum l against its maximum m: -inf where it saw no key, NaN where a score was. */
__device__ __forceinline__ float lse_of(float m, float l, float scale) { return l == 0.f ? NEG_INF : m * scale + logf(l); }
__device__ __forceinline__ float inverse_of(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : l; }

/* The lane's number anew: what follows from it is computed again, a few instructions, where it would hold registers through
   the loop. */
__device__ __forceinline__ int opaque(int lane) {
    asm volatile("" : "+v"(lane));
    return lane;
}

/* wsr_paged_rows.hip: tiles of 32 * rw rows (rw 2 or 4), `blocks` workgroups. */
hipError_t launch_paged_rows(const wsr_paged& p, const PagedPlan& pl, int rw, bool once, int64_t blocks, hipStream_t s);

}  // namespace wsr_serve

#endif
