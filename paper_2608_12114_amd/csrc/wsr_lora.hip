/*
 * wsr_lora.hip - the low-rank adapters of many requests, added to the outputs of shared projections.
 *
 *   y(t) = y0(t) + s_a B_a (A_a x(t)),  a the adapter of token t.
 *
 * Tokens go in tiles of up to 64; more than 64 are first put in the order of their adapters by a kernel
 * of one workgroup.  A tile's work is a list of chunks, eight ranks of one adapter each, over all adapters
 * that its tokens have: whatever the adapters' ranks and however many tokens share one, each chunk's weights
 * are read once per tile.  Two launches over all projections (few tokens over short ones take one, k_lora_small):
 *
 *   k_lora_shrink   (tile, span of the projections' K laid end to end): rows of A from two chunks at a time
 *                   against 16 tokens on v_mfma_f32_16x16x32; a span's sum is stored where the token has the
 *                   row's adapter.
 *   k_lora_expand   (projection, tile, rows): four chunks side by side are the 32 terms of one
 *                   v_mfma_f32_16x16x32; a token's inner vector enters for its own adapter's chunks and as
 *                   zeros for the others; for tokens that were put in order each adapter's chunks lie alike in
 *                   the products, so that a token's sums do not depend on the tile that the order, which is free
 *                   inside an adapter, put it in.  The inner vectors are fp32 (24 bits): they enter as the sum of
 *                   three bf16 terms (24 bits) or of two f16 terms (22 bits, each token's vector scaled by a
 *                   power of two so that its largest entry is near 2^15, the second term by 2^11 more, which
 *                   keeps entries 2^-28 of the largest whole), products with B exact, sums fp32.
 *                   Rounding them to one 16-bit term would leave errors of 2^-9 in the fp32 outputs.
 *
 * Decode is bound by reading the adapters (2 (K + M) rank bytes each): 16 tokens of 14 adapters of 16 ranks over
 * the 8B model, 1.22 GB, take 258 us, 4.7 TB/s (the first launch 95 us at 5.4, the second at 4.5, whose outputs, two
 * streams beside the weights', cost it 60 us).  Prompts are bound by reading and writing the outputs (8 M bytes per
 * token): 2055 tokens of five adapters of 64 ranks over two 14336 x 4096 projections, 526 MB, take 153 us; without
 * the products the second launch alone streams for 100 of them.
 */
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int LT = 256;                        /* threads per workgroup */
constexpr int LW = LT / WAVE;
constexpr int TILE = 64;                       /* tokens of a tile */
constexpr int WINDOW = 64;                     /* ranks worked on at a time */
constexpr int BLOCK_K = 256;                   /* elements of K that a workgroup's waves take in turn, 64 each */
constexpr int SORT_THREADS = 1024;
constexpr int SHRINK_HELD = 512;               /* workgroups on the chip at a time: two per CU */
/* Waves per SIMD of the second launch, a workgroup per CU each: four for up to 16 tokens, three for 64, with units
   of 128 rows (with two, and units of 256 rows, 201 tokens of 31 adapters took 239 us, so 210, 49 of 30 124 and 118;
   with four for 64 tokens the registers spill, and both lose a fifth). */
constexpr int expand_waves(int token_tiles) { return token_tiles == 1 ? 4 : 3; }
typedef u32x4 u32x4_any_t __attribute__((aligned(2)));
typedef u32x2 u32x2_any_t __attribute__((aligned(2)));

struct LoraMod {
    const void *a, *b, *x;
    const float* y0;
    float* y;
    float* v;                                  /* (parts, n_tokens, pitch) partial inner vectors */
    int64_t a_stride, b_stride, x_stride, y0_stride, y_stride, M, K;
    int32_t rank, pitch, parts, block0;        /* pitch: rank up to a multiple of 8; block0: its first block of K */
};
static_assert(sizeof(LoraMod) == 120, "LoraMod layout");

/* Projections and the first unit of work of each, in the launch arguments. */
template <int N>
struct LoraTable {
    int32_t n, units;
    int32_t first[N];
    LoraMod mod[N];
};

struct LoraCall {
    const int32_t *adapter_of, *ranks, *order; /* order: null where tokens are taken as they come */
    const float* scales;
    int32_t n_tokens, n_adapters, tiles;
    int32_t span, slots;                       /* blocks of a shrink workgroup; workgroups that share its rows */
    bool stream;                               /* outputs go past the caches */
};

/* The projection that unit b belongs to: the last whose first unit is <= b. */
template <int N>
__device__ __forceinline__ int mod_of(const LoraTable<N>& tab, int b) {
    const int lane = threadIdx.x % WAVE;
    int m = 0;
#pragma unroll
    for (int i = 0; i < N; i += WAVE) {
        const int j = i + lane;
        m += __builtin_popcountll(__ballot(j < N && j < tab.n && tab.first[j < N ? j : 0] <= b));
    }
    return __builtin_amdgcn_readfirstlane(m) - 1;
}

/* A tile in LDS.  A chunk of its list: adapter << 8 | (eighth of the window) << 4 | ranks it holds (1 to 8, 0 in a
   stand-in). */
template <int COLS>
struct Tile {
    int32_t list[COLS * (WINDOW / 8)];
    int32_t tok[COLS], id[COLS], rank[COLS];   /* -1: no token, no adapter (or none of its ranks) */
    float scale[COLS];
    int32_t chunks, partial;                   /* partial: a chunk under 8 ranks */
};

/* The tile's tokens and the chunks of ranks w0 .. w0 + WINDOW - 1, by the first wave.  PLACED: for
   tokens that were put in order, an adapter's chunks lie where a step of four divides them alike in every tile:
   three or more are filled up to a multiple of four with stand-ins of the last and come first, then pairs, then
   single ones. */
template <bool PLACED, int COLS>
__device__ __forceinline__ void make_tile(const LoraCall& c, int tile, int rank, int w0, Tile<COLS>& t) {
    if (threadIdx.x < WAVE) {
        const int lane = threadIdx.x, at = tile * TILE + lane;
        const bool in = lane < COLS && at < c.n_tokens;
        const int tok = in ? (c.order ? c.order[at] : at) : -1;
        int id = in ? c.adapter_of[tok] : -1, r = 0;
        if (id < 0 || id >= c.n_adapters) id = -1;
        if (id >= 0) {
            r = c.ranks ? min(max(c.ranks[id], 0), rank) : rank;
            if (r == 0) id = -1;
        }
        bool first = id >= 0;                  /* of its adapter in the tile */
        if (c.order) {
            const int before = __shfl_up(id, 1);
            if (lane > 0 && before == id) first = false;
        } else {
            const int n = min(COLS, c.n_tokens);
            for (int j = 0; j < n; ++j)
                if (j < lane && __builtin_amdgcn_readlane(id, j) == id) first = false;
        }
        const int real = first ? (min(max(r - w0, 0), WINDOW) + 7) / 8 : 0;
        const bool placed = PLACED && c.order;
        const int mine = placed && real > 2 ? (real + 3) / 4 * 4 : real;
        int sum = placed && real <= 2 ? 0 : mine;
#pragma unroll
        for (int k = 1; k < WAVE; k <<= 1) {
            const int o = __shfl_up(sum, k);
            if (lane >= k) sum += o;
        }
        int all = __builtin_amdgcn_readlane(sum, WAVE - 1), at_list = sum - mine;
        if (placed) {
            const uint64_t two = __ballot(real == 2), one = __ballot(real == 1), below = (1ull << lane) - 1;
            if (real == 2) at_list = all + 2 * __builtin_popcountll(two & below);
            all += 2 * __builtin_popcountll(two);
            if (real == 1) at_list = all + __builtin_popcountll(one & below);
            all += __builtin_popcountll(one);
        }
        for (int k = 0; k < mine; ++k)
            t.list[at_list + k] = id << 8 | min(k, real - 1) << 4 | (k < real ? min(8, r - w0 - 8 * k) : 0);
        if (lane < COLS) {
            t.tok[lane] = tok, t.id[lane] = id, t.rank[lane] = r;
            t.scale[lane] = id >= 0 && c.scales ? c.scales[id] : 1.f;
        }
        const bool odd = __ballot(first && r % 8) != 0;
        if (lane == 0) t.chunks = all, t.partial = odd;
    }
    __syncthreads();
}

/* 16 bytes of weights, past the caches where a single tile reads them. */
template <bool ONCE>
__device__ __forceinline__ u32x4 load_weights(const char* p) {
    typedef const __attribute__((address_space(1))) u32x4_any_t g_any;
    if constexpr (ONCE) return __builtin_nontemporal_load((g_any*)p);
    else return *(g_any*)p;
}

/* The units of work of a workgroup: a contiguous share of all, so that it meets few projections and makes
   its tile once. */
__device__ __forceinline__ void share_of(int units, int tiles, int& tile, int& u0, int& u1) {
    const int groups = gridDim.x / tiles, i = blockIdx.x / tiles;
    tile = blockIdx.x % tiles;
    u0 = (int)((int64_t)units * i / groups);
    u1 = (int)((int64_t)units * (i + 1) / groups);
}

/* Rows of A are rows of the product and tokens its columns, so what stands in the rows past a chunk's ranks
   or in columns without a token reaches no stored sum: their pointers are set to a valid row.  Past K both
   sides are zeros. */
template <int FMT, int TT, int RT, int N>
__global__ __launch_bounds__(LT) void k_lora_shrink(LoraTable<N> tab, LoraCall c) {
    constexpr int COLS = 16 * TT;
    __shared__ Tile<COLS> t;
    __shared__ f4_t red[LW][RT * TT][WAVE];
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    int made = -1;
    const int tile = blockIdx.x % c.tiles, slot = blockIdx.x / c.tiles % c.slots, span = blockIdx.x / c.tiles / c.slots;
    const int from = span * c.span, to = min(tab.units, from + c.span);
    int m = mod_of(tab, from);
    for (int block = from; block < to; ++m) {
        const LoraMod& d = tab.mod[m];
        const int end = m + 1 < tab.n ? min(to, tab.first[m + 1]) : to;    /* of the blocks in this projection */
        const int part = span - d.block0 / c.span;
        const int k0 = (block - d.block0) * BLOCK_K, k1 = (int)min(d.K, (int64_t)(end - d.block0) * BLOCK_K);
        block = end;
        if (k0 >= k1 && d.K > 0) continue;
        for (int w0 = 0; w0 < d.rank; w0 += WINDOW) {
            if (made != d.rank || d.rank > WINDOW) {
                __syncthreads();
                make_tile<false, COLS>(c, tile, d.rank, w0, t);
                made = d.rank;
            }
            /* a load takes 128 bytes of each of eight rows (eight tokens): lane (g, col) those at 16 (g + 4 (col / 8)) */
            const int lane_at = 16 * (g + col / 8 * 4);
            const char* xr[TT][2];
#pragma unroll
            for (int i = 0; i < TT; ++i)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int tok = t.tok[16 * i + 8 * b + col % 8];
                    xr[i][b] = (const char*)d.x + (tok < 0 ? t.tok[0] : tok) * d.x_stride + lane_at;
                }
            for (int c0 = slot * 2 * RT; c0 < t.chunks; c0 += c.slots * 2 * RT) {
                const char *ar[RT][2], *xp[TT][2];
#pragma unroll
                for (int i = 0; i < TT; ++i) xp[i][0] = xr[i][0], xp[i][1] = xr[i][1];
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int ch = t.list[min(c0 + 2 * i + b, t.chunks - 1)];
                        const int j = w0 + (ch >> 4 & 15) * 8 + min(col % 8, (ch & 15) - 1);
                        ar[i][b] = (const char*)d.a + (ch >> 8) * d.a_stride + j * d.K * 2 + lane_at;
                    }
                f4_t acc[RT][TT] = {};
                /* a batch, 64 elements of every row, is loaded while the one before it is multiplied */
                struct Batch {
                    u32x4 a[RT][2], x[TT][2];
                };
                Batch b0, b1;
                auto load = [&](Batch& b, int ahead) {     /* `ahead` bytes, a constant */
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < RT; ++i) b.a[i][h] = load_weights<TT == 1>(ar[i][h] + ahead);
#pragma unroll
                        for (int i = 0; i < TT; ++i) b.x[i][h] = *(const u32x4*)(xp[i][h] + ahead);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                auto advance = [&](int by) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < RT; ++i) ar[i][h] += by;
#pragma unroll
                        for (int i = 0; i < TT; ++i) xp[i][h] += by;
                    }
                };
                auto multiply = [&](Batch& b) {
#pragma unroll
                    for (int i = 0; i < TT; ++i) wsr::lines_to_slabs(b.x[i][0], b.x[i][1]);
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        wsr::lines_to_slabs(b.a[i][0], b.a[i][1]);
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int j = 0; j < TT; ++j) acc[i][j] = mma16<FMT>(b.a[i][h], b.x[j][h], acc[i][j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                };
                constexpr int B = BLOCK_K / LW, S = BLOCK_K;
                int k = k0 + wave * B;
                advance(k * 2);
                if constexpr (TT > 1) {        /* no registers for two batches */
                    for (; k + B <= k1; k += S) {
                        load(b0, 0);
                        multiply(b0);
                        advance(S * 2);
                    }
                } else if (k + B <= k1) {
                    load(b0, 0);
                    for (; k + 2 * S + B <= k1; k += 2 * S) {
                        load(b1, S * 2);
                        multiply(b0);
                        advance(S * 4);
                        load(b0, 0);
                        multiply(b1);
                    }
                    if (k + S + B <= k1) {
                        load(b1, S * 2);
                        multiply(b0);
                        multiply(b1);
                        k += 2 * S;
                        advance(S * 4);
                    } else {
                        multiply(b0);
                        k += S;
                        advance(S * 2);
                    }
                }
                if (k < k1) {                  /* the last elements, fewer than a batch */
                    const bool in = k + 8 * (g + col / 8 * 4) < k1;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < RT; ++i) b0.a[i][h] = in ? *(const u32x4*)ar[i][h] : wsr::zero4();
#pragma unroll
                        for (int i = 0; i < TT; ++i) b0.x[i][h] = in ? *(const u32x4*)xp[i][h] : wsr::zero4();
                    }
                    multiply(b0);
                }
                __syncthreads();               /* the round before has been read */
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < TT; ++j) red[wave][i * TT + j][lane] = acc[i][j];
                __syncthreads();
                for (int e = wave; e < RT * TT; e += LW) {
                    const int cell = c0 + 2 * (e / TT) + g / 2, token = 16 * (e % TT) + col;
                    if (cell >= t.chunks) continue;
                    const int ch = t.list[cell];
                    if (t.id[token] != ch >> 8) continue;
                    f4_t s = red[0][e][lane];
#pragma unroll
                    for (int w = 1; w < LW; ++w) s += red[w][e][lane];
                    *(f4_t*)(d.v + ((int64_t)part * c.n_tokens + t.tok[token]) * d.pitch + w0 + (ch >> 4 & 15) * 8 + 4 * (g % 2)) = s;
                }
            }
        }
    }
}

/* Eight 16-bit values of a row of B of which `n` count; the others are zeros. */
__device__ __forceinline__ u32x4 load_chunk_row(const char* p, int n) {
    if (n == 8) return *(const u32x4_any_t*)p;
    u32x4 o = wsr::zero4();
    const uint16_t* q = (const uint16_t*)p;
    if (n >= 4) {
        const u32x2 w = *(const u32x2_any_t*)p;
        o.x = w.x, o.y = w.y;
        if (n > 4) o.z = q[4];
        if (n > 5) o.z |= (uint32_t)q[5] << 16;
        if (n > 6) o.w = q[6];
    } else {
        if (n > 0) o.x = q[0];
        if (n > 1) o.x |= (uint32_t)q[1] << 16;
        if (n > 2) o.y = q[2];
    }
    return o;
}

/* Nonzero where one of the eight values is an infinity or NaN (all ones in the exponent). */
template <int FMT>
__device__ __forceinline__ uint32_t not_finite(u32x4 w) {
    constexpr uint32_t E = FMT == WSR_BF16 ? 0x7f807f80u : 0x7c007c00u, ONE = FMT == WSR_BF16 ? 0x00800080u : 0x04000400u;
    return (((w.x & E) + ONE) | ((w.y & E) + ONE) | ((w.z & E) + ONE) | ((w.w & E) + ONE)) & 0x80008000u;
}

/* The values with infinities and NaN as zeros. */
template <int FMT>
__device__ __forceinline__ u32x4 finite_only(u32x4 w) {
    constexpr uint32_t E = FMT == WSR_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= ((w[i] & E) == E ? 0u : 0xffffu) | ((w[i] >> 16 & E) == E ? 0u : 0xffff0000u);
    return w;
}

template <int FMT>
constexpr int terms() { return FMT == WSR_BF16 ? 3 : 2; }
/* What a term after the first is multiplied by.  An f16 residual would fall below the type's smallest steps where an entry
   is far below the token's largest: it gets a power of two of its own, which accumulate() takes off the product. */
template <int FMT>
constexpr float lift() { return FMT == WSR_BF16 ? 1.f : 2048.f; }
/* c + w v_k, term k of the inner vectors. */
template <int FMT>
__device__ __forceinline__ f4_t accumulate(u32x4 w, u32x4 v, f4_t c, int k) {
    if (FMT == WSR_BF16 || k == 0) return mma16<FMT>(w, v, c);
    const f4_t p = mma16<FMT>(w, v, f4_t{0, 0, 0, 0});
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = fmaf(p[e], 1.f / lift<FMT>(), c[e]);
    return c;
}

/* The inner vectors of a window in LDS as 16-bit terms, and the power of two that undoes each token's
   scaling.  A pitch of 16 bytes past a multiple of 128 keeps the 16 tokens' reads on different banks. */
template <int FMT, int COLS>
struct Inner {
    static constexpr int PITCH = terms<FMT>() * WINDOW + 8;
    uint16_t v[COLS * PITCH];
    float undo[COLS];
};

template <int FMT, int COLS>
__device__ __forceinline__ void make_inner(const LoraMod& d, const LoraCall& c, const Tile<COLS>& t, int w0, Inner<FMT, COLS>& in) {
    typedef Inner<FMT, COLS> I;
    const int q = threadIdx.x % 16;            /* sixteen lanes take a token, four ranks each */
    const int pitch = d.pitch;
    auto load = [&](int token, int j) {
        f4_t s = {0, 0, 0, 0};
        const int r = t.id[token] < 0 ? 0 : t.rank[token];
        if (j < r) {
            const float* p = d.v + (int64_t)t.tok[token] * pitch + j;
            const int64_t next = (int64_t)c.n_tokens * pitch;
            int k = 0;
            for (; k + 4 <= d.parts; k += 4, p += 4 * next)
                s += (*(const f4_t*)p + *(const f4_t*)(p + next)) + (*(const f4_t*)(p + 2 * next) + *(const f4_t*)(p + 3 * next));
            if (k + 2 <= d.parts) s += *(const f4_t*)p + *(const f4_t*)(p + next), k += 2, p += 2 * next;
            if (k < d.parts) s += *(const f4_t*)p;
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = j + e < r ? s[e] * t.scale[token] : 0.f;
        }
        return s;
    };
    for (int token = threadIdx.x / 16; token < COLS; token += LT / 16) {
        f4_t s = load(token, w0 + 4 * q);
        if constexpr (FMT == WSR_F16) {
            /* the largest finite entry: beside an infinity the others are still to keep within f16 */
            float top = 0.f;
            auto larger = [&](f4_t o) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fabsf(o[e]) < __builtin_inff() ? fmaxf(top, fabsf(o[e])) : top;
            };
            if (d.rank <= WINDOW) larger(s);
            else
                for (int w = 0; w < d.rank; w += WINDOW) larger(load(token, w + 4 * q));
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
            /* 2^14 <= scaled top < 2^15, the exponent kept where both powers of two are normal */
            const int e = top > 0.f ? min(max(15 - __builtin_amdgcn_frexp_expf(top), -126), 126) : 0;
            s *= __builtin_amdgcn_ldexpf(1.f, e);
            if (q == 0) in.undo[token] = __builtin_amdgcn_ldexpf(1.f, -e);
        }
#pragma unroll
        for (int k = 0; k < terms<FMT>(); ++k) {
            typedef typename Half<FMT>::t H;
            u32x2 w;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                w[e] = pack2<FMT>(s[2 * e], s[2 * e + 1]);
                const float a = s[2 * e] - (float)(H)s[2 * e], b = s[2 * e + 1] - (float)(H)s[2 * e + 1];
                s[2 * e] = a == a ? a * lift<FMT>() : 0.f, s[2 * e + 1] = b == b ? b * lift<FMT>() : 0.f;   /* inf - inf */
            }
            *(u32x2*)(in.v + token * I::PITCH + k * WINDOW + 4 * q) = w;
        }
    }
    __syncthreads();
}

/* A wave's 16 RW rows of a unit against the tile's tokens, U steps of four chunks at a time.  STREAM: outputs are
   loaded and stored past the caches. */
template <int FMT, int TT, int RW, bool STREAM, int N>
__global__ __launch_bounds__(LT) __attribute__((amdgpu_waves_per_eu(expand_waves(TT)))) void k_lora_expand(LoraTable<N> tab, LoraCall c) {
    constexpr int COLS = 16 * TT, ROWS = LW * 16 * RW, U = TT == 1 ? 4 : 2, NTERM = terms<FMT>();
    typedef Inner<FMT, COLS> I;
    __shared__ Tile<COLS> t;
    __shared__ I in;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    int tile, u0, u1, made = -1, inner = -1;
    share_of(tab.units, c.tiles, tile, u0, u1);
    if (u0 >= u1) return;
    const int used = min(TT, (c.n_tokens - tile * TILE + 15) / 16);    /* token tiles that hold tokens */
    /* Outputs are read and written as whole 128-byte lines: the sums of two 16-row tiles change places so that one
       access takes both tiles of eight tokens (col / 8 the tile), the next those of the other eight.  Access i: */
    auto out_col = [&](int i) { return RW > 1 ? i % 2 * 8 + col % 8 : col; };
    auto out_row = [&](int i) { return RW > 1 ? i / 2 * 32 + col / 8 * 16 + 4 * g : 16 * i + 4 * g; };
    int m = mod_of(tab, u0);
    for (int unit = u0; unit < u1; ++unit) {
        while (m + 1 < tab.n && tab.first[m + 1] <= unit) ++m;
        const LoraMod& d = tab.mod[m];
        const int64_t i0 = (int64_t)(unit - tab.first[m]) * ROWS + wave * 16 * RW;
        const bool whole = i0 + 16 * RW <= d.M;
        f4_t acc[RW][TT] = {}, y0[RW][TT];
        for (int w0 = 0; w0 < d.rank; w0 += WINDOW) {
            if (made != d.rank || d.rank > WINDOW) {
                __syncthreads();
                make_tile<true, COLS>(c, tile, d.rank, w0, t);
                made = d.rank;
            }
            if (w0 == 0 && whole && d.y0) {
#pragma unroll
                for (int j = 0; j < TT; ++j)
#pragma unroll
                    for (int i = 0; i < RW; ++i) {
                        const int tok = t.tok[16 * j + out_col(i)];
                        const float* src = (const float*)((const char*)d.y0 + (tok < 0 ? t.tok[0] : tok) * d.y0_stride);
                        if constexpr (STREAM) y0[i][j] = __builtin_nontemporal_load((const f4_any_t*)(src + i0 + out_row(i)));
                        else y0[i][j] = *(const f4_any_t*)(src + i0 + out_row(i));
                    }
            }
            if (t.chunks == 0) break;          /* no adapter reaches this window or a later one */
            if (inner != m || d.rank > WINDOW) {
                __syncthreads();
                make_inner<FMT, COLS>(d, c, t, w0, in);
                inner = m;
            }
            int id[TT];
#pragma unroll
            for (int j = 0; j < TT; ++j) id[j] = t.id[16 * j + col];
            const bool partial = __builtin_amdgcn_readfirstlane(t.partial);
            const int chunks = __builtin_amdgcn_readfirstlane(t.chunks);
            int64_t row[RW];
#pragma unroll
            for (int i = 0; i < RW; ++i) row[i] = min(i0 + 16 * i + col, d.M - 1) * d.rank * 2;
            /* U steps of four chunks, all loads before the products */
            auto batch = [&](auto steps, int c0) {
                constexpr int U = decltype(steps)::value;
                int adapter[U], ch[U];
                u32x4 b[U][RW];
                const char* p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {  /* past the list's end the last chunk stands in, against no token */
                    const int cell = c0 + 4 * u + g;
                    ch[u] = t.list[min(cell, chunks - 1)];
                    p[u] = (const char*)d.b + (ch[u] >> 8) * d.b_stride + (w0 + (ch[u] >> 4 & 15) * 8) * 2;
                    adapter[u] = cell < chunks && ch[u] & 15 ? ch[u] >> 8 : -2;
                }
                if (partial) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < RW; ++i) b[u][i] = load_chunk_row(p[u] + row[i], ch[u] & 15);
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int i = 0; i < RW; ++i) b[u][i] = load_weights<TT == 1>(p[u] + row[i]);
                }
                __builtin_amdgcn_sched_barrier(0);
                /* zero times an infinity or NaN of one adapter's weights would reach the tokens of the others, and a second
                   term of the other sign make NaN of an infinity: such steps go adapter by adapter, its sums taken over
                   by its own tokens only and its infinities and NaN multiplied with the first terms */
                uint32_t apart = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    uint32_t bad = 0;
#pragma unroll
                    for (int i = 0; i < RW; ++i) bad |= not_finite<FMT>(b[u][i]);
                    apart |= __ballot(bad != 0) ? 1u << u : 0u;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (TT > 1 && c0 + 4 * u >= chunks) break;
                    const int chunk = (ch[u] >> 4 & 15) * 8;
#pragma unroll
                    for (int j = 0; j < TT; ++j) {
                        if (j >= used) break;
                        const bool own = id[j] == adapter[u];
                        if (__ballot(own) == 0) continue;
                        u32x4 v[NTERM];
#pragma unroll
                        for (int k = 0; k < NTERM; ++k) {
                            v[k] = *(const u32x4*)(in.v + (16 * j + col) * I::PITCH + k * WINDOW + chunk);
                            if (!own) v[k] = wsr::zero4();
                        }
                        if (!(apart >> u & 1)) {
#pragma unroll
                            for (int k = 0; k < NTERM; ++k)
#pragma unroll
                                for (int i = 0; i < RW; ++i) acc[i][j] = accumulate<FMT>(b[u][i], v[k], acc[i][j], k);
                        } else {
#pragma unroll 1
                            for (int o = 0; o < 4; ++o) {
                                const int its = __shfl(adapter[u], 16 * o);
                                if (o && its == __shfl(adapter[u], 16 * (o - 1))) continue;
                                const bool mine = id[j] >= 0 && id[j] == its;
#pragma unroll
                                for (int i = 0; i < RW; ++i) {
                                    f4_t s = acc[i][j];
                                    u32x4 w = adapter[u] == its ? b[u][i] : wsr::zero4();
                                    asm volatile("" : "+v"(w));          /* or the next line's registers are held all along */
#pragma unroll
                                    for (int k = 0; k < NTERM; ++k) {
                                        s = accumulate<FMT>(w, v[k], s, k);
                                        if (k == 0) w = finite_only<FMT>(w);   /* later terms may differ in sign */
                                    }
#pragma unroll
                                    for (int e = 0; e < 4; ++e) acc[i][j][e] = mine ? s[e] : acc[i][j][e];
                                }
                            }
                        }
                    }
                }
            };
            if constexpr (TT > 1) {            /* few steps at a time: the last may be half empty */
                for (int c0 = 0; c0 < chunks; c0 += 4 * U) batch(std::integral_constant<int, U>{}, c0);
            } else {
                int c0 = 0;
                for (; c0 + 4 * (U - 1) < chunks; c0 += 4 * U) batch(std::integral_constant<int, U>{}, c0);
                if (c0 + 4 < chunks) batch(std::integral_constant<int, 2>{}, c0), c0 += 8;
                if (c0 < chunks) batch(std::integral_constant<int, 1>{}, c0);
            }
        }
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            if constexpr (FMT == WSR_F16) {
                const float undo = t.id[16 * j + col] >= 0 ? in.undo[16 * j + col] : 1.f;
#pragma unroll
                for (int i = 0; i < RW; ++i) acc[i][j] *= undo;
            }
            if constexpr (RW > 1) {
#pragma unroll
                for (int i = 0; i < RW; i += 2) {
                    u32x4 a = __builtin_bit_cast(u32x4, acc[i][j]), b = __builtin_bit_cast(u32x4, acc[i + 1][j]);
                    wsr::lines_to_slabs(a, b);
                    acc[i][j] = __builtin_bit_cast(f4_t, a), acc[i + 1][j] = __builtin_bit_cast(f4_t, b);
                }
            }
#pragma unroll
            for (int i = 0; i < RW; ++i) {
                const int cell = 16 * j + out_col(i), tok = t.tok[cell];
                const bool has = t.id[cell] >= 0;
                if (tok < 0 || (!has && d.y0 == d.y)) continue;
                const int64_t at = i0 + out_row(i);
                float* dst = (float*)((char*)d.y + tok * d.y_stride) + at;
                f4_t s = acc[i][j];
                if (whole) {
                    if (d.y0) s = has ? y0[i][j] + s : y0[i][j];
                    if constexpr (STREAM) __builtin_nontemporal_store(s, (f4_any_t*)dst);
                    else *(f4_any_t*)dst = s;
                } else {
                    const float* src = d.y0 ? (const float*)((const char*)d.y0 + tok * d.y0_stride) + at : nullptr;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (at + k < d.M) dst[k] = !src ? s[k] : has ? src[k] + s[k] : src[k];
                }
            }
        }
    }
}

/* Few tokens over few projections, in one launch: a workgroup takes LT rows of a projection, works out the inner
   vectors for itself (a wave four rows of A at a time, on the vector ALUs) and gives each thread a row of B, whose
   loads are under way before.  Bound by one pass of latency: 1 token, 4096 x 4096, 16 ranks 6.1 us in a graph, 10.2
   in two launches. */
constexpr int SMALL_RANK = WINDOW;
template <int FMT, int N>
__global__ __launch_bounds__(LT) void k_lora_small(LoraTable<N> tab, LoraCall c) {
    constexpr int RJ = 4, U = 4, PIECES = SMALL_RANK / 8;
    __shared__ float v[2][SMALL_RANK];
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block();
    const int m = mod_of(tab, blockIdx.x);
    const LoraMod& d = tab.mod[m];
    const int64_t row = (int64_t)(blockIdx.x - tab.first[m]) * LT + threadIdx.x;
    int half = 0;
    for (int t = 0; t < c.n_tokens; ++t) {
        int id = c.adapter_of[t], r = 0;
        if (id >= 0 && id < c.n_adapters) r = c.ranks ? min(max(c.ranks[id], 0), d.rank) : d.rank;
        if (r == 0 && d.y0 == d.y) continue;
        float* y = (float*)((char*)d.y + t * d.y_stride) + row;
        float s = d.y0 && row < d.M ? ((const float*)((const char*)d.y0 + t * d.y0_stride))[row] : 0.f;
        if (r > 0) {
            const char* br = (const char*)d.b + id * d.b_stride + min(row, d.M - 1) * d.rank * 2;
            u32x4 b[PIECES];
#pragma unroll
            for (int p = 0; p < PIECES; ++p) b[p] = 8 * p < r ? load_chunk_row(br + 16 * p, min(8, r - 8 * p)) : wsr::zero4();
            const char *ar = (const char*)d.a + id * d.a_stride, *xr = (const char*)d.x + t * d.x_stride;
            const float scale = c.scales ? c.scales[id] : 1.f;
            for (int j = wave * RJ; j < r; j += LW * RJ) {
                const char* a[RJ];
                float acc[RJ] = {};
#pragma unroll
                for (int i = 0; i < RJ; ++i) a[i] = ar + min(j + i, r - 1) * d.K * 2;
                auto step = [&](auto steps, int64_t k) {
                    constexpr int S = decltype(steps)::value;
                    u32x4 x[S], w[S][RJ];
#pragma unroll
                    for (int u = 0; u < S; ++u) {
                        x[u] = *(const u32x4*)(xr + (k + u * WAVE * 8) * 2);
#pragma unroll
                        for (int i = 0; i < RJ; ++i) w[u][i] = *(const u32x4*)(a[i] + (k + u * WAVE * 8) * 2);
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int u = 0; u < S; ++u) {
                        float xv[8];
                        unpack8<FMT>(x[u], xv);
#pragma unroll
                        for (int i = 0; i < RJ; ++i) {
                            float wv[8];
                            unpack8<FMT>(w[u][i], wv);
#pragma unroll
                            for (int e = 0; e < 8; ++e) acc[i] = fmaf(wv[e], xv[e], acc[i]);
                        }
                    }
                };
                int64_t k = lane * 8;
                for (; k + (U - 1) * WAVE * 8 < d.K; k += U * WAVE * 8) step(std::integral_constant<int, U>{}, k);
                for (; k < d.K; k += WAVE * 8) step(std::integral_constant<int, 1>{}, k);
#pragma unroll
                for (int i = 0; i < RJ; ++i) {
                    const float sum = wsr::wave_sum(acc[i]);
                    if (lane == 0 && j + i < r) v[half][j + i] = sum * scale;
                }
            }
            __syncthreads();                   /* the next vector goes to the other half */
            float dot = 0.f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                if (8 * p >= r) break;
                float bv[8];
                unpack8<FMT>(b[p], bv);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (8 * p + e < r) dot = fmaf(bv[e], v[half][8 * p + e], dot);
            }
            s += dot;
            half ^= 1;
        }
        if (row < d.M) *y = s;
    }
}

/* Tokens in the order of their adapters, those without one last.  The order inside an adapter follows from
   the atomics and may differ from run to run; a token's results depend neither on its place in a tile nor on
   the tile. */
__global__ __launch_bounds__(SORT_THREADS) void k_lora_sort(const int32_t* adapter_of, int n_tokens, int n_adapters,
                                                            int32_t* order) {
    extern __shared__ int32_t bin[];           /* [n_adapters + 1] */
    __shared__ int32_t sc[SORT_THREADS / WAVE];
    const int n = n_adapters + 1, tid = threadIdx.x;
    for (int i = tid; i < n; i += SORT_THREADS) bin[i] = 0;
    __syncthreads();
    for (int t = tid; t < n_tokens; t += SORT_THREADS) {
        const int id = adapter_of[t];
        atomicAdd(&bin[id >= 0 && id < n_adapters ? id : n_adapters], 1);
    }
    __syncthreads();
    const int per = (n + SORT_THREADS - 1) / SORT_THREADS, b0 = min(n, tid * per), b1 = min(n, b0 + per);
    int tokens = 0;
    for (int i = b0; i < b1; ++i) tokens += bin[i];
    int at = tokens;                           /* of the threads before: inside the wave, then of the waves before */
#pragma unroll
    for (int k = 1; k < WAVE; k <<= 1) {
        const int o = __shfl_up(at, k);
        if (tid % WAVE >= k) at += o;
    }
    if (tid % WAVE == WAVE - 1) sc[tid / WAVE] = at;
    at -= tokens;
    __syncthreads();
    for (int w = 0; w < tid / WAVE; ++w) at += sc[w];
    for (int i = b0; i < b1; ++i) {
        const int count = bin[i];
        bin[i] = at;
        at += count;
    }
    __syncthreads();
    for (int t = tid; t < n_tokens; t += SORT_THREADS) {
        const int id = adapter_of[t];
        order[atomicAdd(&bin[id >= 0 && id < n_adapters ? id : n_adapters], 1)] = t;
    }
}

/* ---- host ------------------------------------------------------------------------------------------ */

static int tiles_of(int32_t n_tokens) { return (n_tokens + TILE - 1) / TILE; }

static int64_t blocks_of(const wsr_lora& m) { return std::max<int64_t>(1, (m.K + BLOCK_K - 1) / BLOCK_K); }

/* A run: the next projections of a call that one pair of launches takes, of one type and at most a table's length.  Those
   without rows (M = 0), whose pointers may be null, are in no run: no launch and no workspace knows of them. */
constexpr int TABLE_MAX = 224;
struct Run {
    const wsr_lora* mod[TABLE_MAX];
    int32_t n = 0;
};
/* Fills the run from projection i on; the projection that the next begins with. */
static int32_t take_run(const wsr_lora* mods, int32_t i, int32_t n, Run& run) {
    run.n = 0;
    for (; i < n; ++i) {
        if (mods[i].M == 0) continue;
        if (run.n == TABLE_MAX || (run.n && mods[i].fmt != run.mod[0]->fmt)) break;
        run.mod[run.n++] = &mods[i];
    }
    return i;
}

/* Blocks of K of a shrink workgroup's span at least: spans that give every workgroup the chip holds (two per CU) an
   equal share, of two blocks or more; for many tokens so long that a token's parts, which the second launch adds
   up once per workgroup and projection, stay within 2 KiB. */
static int least_span(const Run& run, int32_t n_tokens) {
    int64_t all = 0, least = 2;
    for (int32_t i = 0; i < run.n; ++i) {
        all += blocks_of(*run.mod[i]);
        if (n_tokens > TILE) least = std::max(least, blocks_of(*run.mod[i]) / std::max(1, 512 / run.mod[i]->rank));
    }
    const int64_t held = std::max<int64_t>(1, SHRINK_HELD / tiles_of(n_tokens));
    return (int)std::min<int64_t>(1 << 24, std::max(least, (all + held - 1) / held));
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }
static size_t order_bytes(int32_t n_tokens) { return n_tokens <= TILE ? 0 : up256(4 * (size_t)n_tokens); }
constexpr int64_t SMALL_BYTES[] = {448 << 10, 256 << 10, 192 << 10}, SMALL_TOKENS = 3, SMALL_UNITS = 512;

/* Places a run's projections: blocks, parts and partial inner vectors; the bytes of the latter, enough for spans of
   `least` blocks or more. */
static size_t place(const Run& run, int32_t n_tokens, int least, int span, LoraMod* out, char* ws) {
    int64_t block = 0;
    size_t bytes = 0;
    for (int32_t i = 0; i < run.n; ++i) {
        const wsr_lora& m = *run.mod[i];
        const int64_t count = blocks_of(m), last = block + count - 1;
        const int pitch = (m.rank + 7) / 8 * 8;
        if (out)
            out[i] = LoraMod{m.a, m.b, m.x, m.y0, m.y, reinterpret_cast<float*>(ws + bytes), m.a_stride, m.b_stride,
                             m.x_tok_stride, m.y0_tok_stride, m.y_tok_stride, m.M, m.K, m.rank, pitch,
                             (int)(last / span - block / span + 1), (int32_t)block};
        bytes += up256((size_t)((count + least - 2) / least + 1) * n_tokens * pitch * 4);
        block = last + 1;
    }
    return bytes;
}

size_t lora_workspace(const wsr_lora* mods, int32_t n, int32_t n_tokens) {
    size_t most = 256;                         /* the runs follow one another and share it */
    Run run;
    for (int32_t i = 0; (i = take_run(mods, i, n, run)), run.n;) {
        const int least = least_span(run, n_tokens);
        most = std::max(most, place(run, n_tokens, least, least, nullptr, nullptr));
    }
    return order_bytes(n_tokens) + most;
}

/* Workgroups of a launch: one per unit and tile, or as many as the chip holds at a time, each with an equal
   share. */
static unsigned grid_of(int64_t units, int64_t tiles, int64_t held) {
    return (unsigned)(tiles * std::max<int64_t>(1, std::min(units, held / tiles)));
}

template <int FMT, int TT, int RW, bool STREAM, int N>
static hipError_t launch_expand(LoraTable<N>& tab, const LoraCall& c, hipStream_t s) {
    constexpr int ROWS = LW * 16 * RW;
    int64_t units = 0;
    for (int i = 0; i < tab.n; ++i) {
        tab.first[i] = (int32_t)units;
        units += (tab.mod[i].M + ROWS - 1) / ROWS;
        if (units > INT32_MAX) return hipErrorInvalidValue;
    }
    if (units == 0) return hipSuccess;
    tab.units = (int32_t)units;
    hipLaunchKernelGGL((k_lora_expand<FMT, TT, RW, STREAM, N>), dim3(grid_of(units, c.tiles, 256 * expand_waves(TT))), dim3(LT), 0, s, tab, c);
    return hipGetLastError();
}

template <int FMT, int TT, int N>
static hipError_t launch_pair(LoraTable<N>& tab, const LoraCall& c, bool one, hipStream_t s) {
    int64_t rows = 0;
    for (int i = 0; i < tab.n; ++i) tab.first[i] = tab.mod[i].block0, rows += tab.mod[i].M;
    const int64_t blocks = (int64_t)tab.units, spans = (blocks + c.span - 1) / c.span;
    if (spans * c.tiles * c.slots > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(spans * c.tiles * c.slots));
    if (one) hipLaunchKernelGGL((k_lora_shrink<FMT, 1, 1, N>), grid, dim3(LT), 0, s, tab, c);
    else hipLaunchKernelGGL((k_lora_shrink<FMT, TT, 4, N>), grid, dim3(LT), 0, s, tab, c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    /* units of 64 rows instead of 128 where the latter would take less than three eighths of the chip's 1024 places (16
       tokens of 14 adapters, 64 and 128: 43008 rows 25.3 and 26.1 us, 57344 23.2 and 22.5, 86016 37.3 and 33.1; 4 tokens
       of 64 ranks, 40960 rows 22.4 and 23.0, 61440 28.0 and 27.4) */
    if constexpr (TT == 1)
        if (rows / 128 < 384) return launch_expand<FMT, 1, 1, false, N>(tab, c, s);
    if (c.stream) return launch_expand<FMT, TT, 2, true, N>(tab, c, s);
    return launch_expand<FMT, TT, 2, false, N>(tab, c, s);
}

/* Whether one launch does: every workgroup reads all of the tokens' rows of A, so they are to be short, the workgroups few
   and the tokens, which go one after the other, few.  By the bytes of A that a workgroup reads, one launch and two (us):
   1 token 128 KiB 6.1 and 10.1, 256 KiB 9.4 and 12.5, 448 KiB 11.2 and 11.7, 512 KiB 13.4 and 13.0; 2 tokens 256 KiB 10.1
   and 12.2, 290 KiB 20.4 and 15.8; 3 tokens 192 KiB 11.4 and 12.2, 217 KiB 14.9 and 15.2, 240 KiB 13.3 and 10.5. */
static bool is_small(const LoraMod* mods, int n, int32_t n_tokens) {
    if (n_tokens > SMALL_TOKENS) return false;
    int64_t units = 0;
    for (int i = 0; i < n; ++i) {
        if (mods[i].rank > SMALL_RANK || n_tokens * mods[i].rank * mods[i].K * 2 > SMALL_BYTES[n_tokens - 1]) return false;
        units += (mods[i].M + LT - 1) / LT;
    }
    return units <= SMALL_UNITS;
}

template <int FMT, int N>
static hipError_t launch_small(LoraTable<N>& tab, const LoraCall& c, hipStream_t s) {
    int64_t units = 0;
    for (int i = 0; i < tab.n; ++i) {
        tab.first[i] = (int32_t)units;
        units += (tab.mod[i].M + LT - 1) / LT;
    }
    if (units == 0) return hipSuccess;
    hipLaunchKernelGGL((k_lora_small<FMT, N>), dim3((unsigned)units), dim3(LT), 0, s, tab, c);
    return hipGetLastError();
}

template <int N>
static hipError_t launch_table(const LoraMod* mods, int n, int fmt, int64_t blocks, const LoraCall& c, bool one, hipStream_t s) {
    LoraTable<N> tab;
    tab.n = n;
    tab.units = (int32_t)blocks;
    std::copy(mods, mods + n, tab.mod);
    if constexpr (N == 8)
        if (is_small(mods, n, c.n_tokens))
            return fmt == WSR_F16 ? launch_small<WSR_F16, N>(tab, c, s) : launch_small<WSR_BF16, N>(tab, c, s);
    const bool few = c.n_tokens <= 16;
    if (fmt == WSR_F16) return few ? launch_pair<WSR_F16, 1, N>(tab, c, one, s) : launch_pair<WSR_F16, 4, N>(tab, c, one, s);
    return few ? launch_pair<WSR_BF16, 1, N>(tab, c, one, s) : launch_pair<WSR_BF16, 4, N>(tab, c, one, s);
}

hipError_t launch_lora(const wsr_lora* mods, int32_t n, int32_t n_tokens, const int32_t* adapter_of, int32_t n_adapters,
                       const int32_t* ranks, const float* scales, void* ws, hipStream_t s) {
    Run run;
    int32_t next = take_run(mods, 0, n, run);
    if (run.n == 0) return hipSuccess;         /* no outputs */
    char* at = static_cast<char*>(ws);
    LoraCall c{};
    c.adapter_of = adapter_of, c.ranks = ranks, c.scales = scales, c.n_tokens = n_tokens, c.n_adapters = n_adapters;
    c.tiles = tiles_of(n_tokens);
    if (n_tokens > TILE) {
        int32_t* order = reinterpret_cast<int32_t*>(at);
        at += order_bytes(n_tokens);
        c.order = order;
        hipLaunchKernelGGL(k_lora_sort, dim3(1), dim3(SORT_THREADS), 4 * ((size_t)n_adapters + 1), s, adapter_of, n_tokens,
                           n_adapters, order);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    LoraMod placed[TABLE_MAX];
    for (; run.n; next = take_run(mods, next, n, run)) {
        const int fmt = run.mod[0]->fmt;
        int64_t blocks = 0;
        int rank = 0;
        for (int32_t j = 0; j < run.n; ++j) blocks += blocks_of(*run.mod[j]), rank = std::max(rank, run.mod[j]->rank);
        if (blocks > INT32_MAX) return hipErrorInvalidValue;
        /* chunks that a tile can have, and rounds of four 16-row tiles, two chunks each; one such tile is
           enough for a single adapter of 16 ranks (7.4 us with four, so 6.0) */
        const int64_t chunks = (int64_t)std::min(std::min(n_tokens, TILE), std::max(1, n_adapters)) * ((std::min(rank, WINDOW) + 7) / 8);
        const bool one = n_tokens <= 16 && chunks <= 2;
        const int64_t rounds = one ? 1 : (chunks + 7) / 8;
        /* a round's loads and sums pay from about eight blocks on: where the chip's share is less, several
           workgroups take a longer span and its rounds in turn (`slots`), and where it is more than the call has,
           the rounds are spread over what is left */
        const int least = least_span(run, n_tokens);
        c.slots = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, 8 / least));
        /* outputs larger than the chip's second-level caches are gone from them before they are read again: loaded and
           stored past them (16 tokens over the 8B model 277 us, so 258; 2055 prompt tokens 160 and 154) */
        int64_t rows = 0;
        for (int32_t j = 0; j < run.n; ++j) rows += run.mod[j]->M;
        c.stream = rows * n_tokens * 4 >= 32 << 20;
        const int64_t held = std::max<int64_t>(1, SHRINK_HELD / c.tiles);
        c.span = (int32_t)std::max<int64_t>(least, std::min<int64_t>(8, (blocks * c.slots + held - 1) / held));
        const int64_t spans = (blocks + c.span - 1) / c.span;
        c.slots = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, held / spans));
        place(run, n_tokens, least, c.span, placed, at);
        const hipError_t e = run.n <= 8 ? launch_table<8>(placed, run.n, fmt, blocks, c, one, s)
                                    : launch_table<TABLE_MAX>(placed, run.n, fmt, blocks, c, one, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace wsr_step
