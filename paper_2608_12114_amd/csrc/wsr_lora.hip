/*
 * wsr_lora.hip - the low-rank adapters of many requests, added to the outputs of shared projections.
 *
 *   y(t) = y0(t) + s_a B_a (A_a x(t)),  a the adapter of token t.
 *
 * Tokens of one adapter are taken together in tiles, so that an adapter's weights are read once per
 * tile: up to 64 tokens, each workgroup finds its tile from the adapter numbers by ballot; more
 * tokens are sorted by a kernel of one workgroup first.  Then two launches over all projections:
 *
 *   k_lora_shrink   (projection, tile, 64 ranks, part of K): A x on v_mfma_f32_16x16x32, the part's sums
 *                   to the workspace in fp32 (parts keep a single projection spread over the chip)
 *   k_lora_expand   (projection, tile, 256 rows): the parts summed and scaled, then B (A x) on
 *                   v_mfma_f32_16x16x4_f32: B's 16-bit values are exact in fp32 and the inner vector
 *                   keeps its 24 bits, which a 16-bit instruction would cut to 8 or 11
 *
 * Decode is bound by reading the adapters (2 (K + M) rank bytes each), prompts by reading and
 * writing the outputs (8 M bytes per token).
 */
#include <hip/hip_runtime.h>

#include <algorithm>

#include "wsr_step_device.h"

namespace wsr_step {

constexpr int LT = 256;                        /* threads per workgroup */
constexpr int LW = LT / WAVE;
constexpr int BALLOT_TOKENS = 64;              /* up to here tiles are found by ballot */
constexpr int EXPAND_ROWS = 256;               /* rows of a workgroup: 64 per wave */
constexpr int RANKS = 64;                      /* ranks of a shrink workgroup */
constexpr int SORT_THREADS = 1024;
constexpr int MAX_ADAPTERS = 8192;

struct LoraMod {
    const void *a, *b, *x;
    const float* y0;
    float* y;
    float* v;                                  /* (parts, n_tokens, pitch) partial inner vectors */
    int64_t a_stride, b_stride, x_stride, y0_stride, y_stride, M, K;
    int32_t rank, pitch, parts, part_k;        /* pitch: rank up to a multiple of 16 */
};
static_assert(sizeof(LoraMod) == 120, "LoraMod layout");

/* Projections and the first workgroup of each, in the launch arguments. */
template <int N>
struct LoraTable {
    int32_t n;
    int32_t first[N];
    LoraMod mod[N];
};

struct LoraCall {
    const int32_t *adapter_of, *ranks, *tiles; /* tiles: null by ballot; else count, then (adapter, first, tokens), then the order */
    const float* scales;
    const int32_t* order;
    int32_t n_tokens, n_adapters, tile_slots;  /* tiles of the grid per projection */
};

/* The projection that workgroup b belongs to: the last whose first workgroup is <= b. */
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

/* Tile `tile` of the call: its adapter, rank and tokens (toks, -1 beyond them); false if there is none. */
template <int COLS>
__device__ __forceinline__ bool find_tile(const LoraCall& c, int tile, int rank, int (&toks)[COLS], int& adapter, int& r) {
    const int lane = threadIdx.x % WAVE;
    int count;
    if (!c.tiles) {
        const int id = lane < c.n_tokens ? c.adapter_of[lane] : -2;
        const bool has = id >= 0 && id < c.n_adapters;
        const int key = lane < c.n_tokens ? (has ? id : -1) : -2;
        adapter = __builtin_amdgcn_readlane(key, tile);
        const uint64_t mine = __ballot(key == adapter);
        const int before = __builtin_popcountll(mine & ((1ull << tile) - 1));
        if (before % COLS) return false;              /* not the first token of a tile */
        const int at = __builtin_popcountll(mine & ((1ull << lane) - 1)) - before;
        count = min(COLS, (int)__builtin_popcountll(mine) - before);
        if (threadIdx.x < WAVE) {
            if (lane < COLS) toks[lane] = -1;
            if (key == adapter && at >= 0 && at < COLS) toks[at] = lane;
        }
    } else {
        if (tile >= c.tiles[0]) return false;
        adapter = __builtin_amdgcn_readfirstlane(c.tiles[1 + 3 * tile]);
        const int first = c.tiles[2 + 3 * tile];
        count = c.tiles[3 + 3 * tile];
        for (int i = threadIdx.x; i < COLS; i += LT) toks[i] = i < count ? c.order[first + i] : -1;
    }
    r = adapter < 0 ? 0 : c.ranks ? min(max(c.ranks[adapter], 0), rank) : rank;
    r = __builtin_amdgcn_readfirstlane(r);
    __syncthreads();
    return true;
}

template <int FMT, int NT, int N>
__global__ __launch_bounds__(LT) void k_lora_shrink(LoraTable<N> tab, LoraCall c) {
    constexpr int RT = RANKS / 16;
    __shared__ int toks[16 * NT];
    __shared__ f4_t red[LW][RT * NT][WAVE];
    const int m = mod_of(tab, blockIdx.x);
    const LoraMod& d = tab.mod[m];
    int at = blockIdx.x - tab.first[m];
    const int part = at % d.parts;
    at /= d.parts;
    const int blocks = (d.rank + RANKS - 1) / RANKS, r0 = at % blocks * RANKS, tile = at / blocks;
    int adapter, r;
    if (!find_tile<16 * NT>(c, tile, d.rank, toks, adapter, r) || r0 >= r) return;
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    const char* a = (const char*)d.a + adapter * d.a_stride;
    const int64_t k0 = (int64_t)part * d.part_k, k1 = min(d.K, k0 + d.part_k);
    const char* xr[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) xr[t] = toks[16 * t + col] < 0 ? nullptr : (const char*)d.x + toks[16 * t + col] * d.x_stride;
    const int tiles_r = (min(RANKS, r - r0) + 15) / 16;
    f4_t acc[RT][NT] = {};
    for (int64_t k = k0 + wave * 32; k < k1; k += 32 * LW) {
        const int64_t kk = k + 8 * g;
        u32x4 xv[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) xv[t] = kk < k1 && xr[t] ? *(const u32x4*)(xr[t] + kk * 2) : wsr::zero4();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            if (i >= tiles_r) break;
            const int j = r0 + 16 * i + col;
            const u32x4 av = kk < k1 && j < r ? *(const u32x4*)(a + (j * d.K + kk) * 2) : wsr::zero4();
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[i][t] = mma_16x16x32<FMT>(av, xv[t], acc[i][t]);
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) red[wave][i * NT + t][lane] = acc[i][t];
    __syncthreads();
    for (int e = wave; e < tiles_r * NT; e += LW) {
        const int i = e / NT, t = e % NT, tok = toks[16 * t + col];
        f4_t s = red[0][e][lane];
#pragma unroll
        for (int w = 1; w < LW; ++w) s += red[w][e][lane];
        if (tok >= 0) *(f4_t*)(d.v + ((int64_t)part * c.n_tokens + tok) * d.pitch + r0 + 16 * i + 4 * g) = s;
    }
}

/* Four consecutive 16-bit values of a row of B as fp32, those from `left` on as zeros. */
template <int FMT>
__device__ __forceinline__ f4_t load_b4(const char* p, int left, bool wide) {
    if (left <= 0) return f4_t{0, 0, 0, 0};
    uint32_t w0 = 0, w1 = 0;
    if (wide && left >= 4) {
        const u32x2 w = *(const u32x2*)p;
        w0 = w.x, w1 = w.y;
    } else {
        const uint16_t* q = (const uint16_t*)p;
        w0 = q[0];
        if (left > 1) w0 |= (uint32_t)q[1] << 16;
        if (left > 2) w1 = q[2];
        if (left > 3) w1 |= (uint32_t)q[3] << 16;
    }
    float o0, o1, o2, o3;
    unpack2<FMT>(w0, o0, o1);
    unpack2<FMT>(w1, o2, o3);
    return f4_t{o0, o1, o2, o3};
}

constexpr int VRANKS = 128;                    /* ranks of the inner vectors held in LDS at a time */
constexpr int VPAD = 4;                        /* floats between their rows */

template <int FMT, int NT, int N>
__global__ __launch_bounds__(LT) void k_lora_expand(LoraTable<N> tab, LoraCall c) {
    __shared__ float vs[16 * NT * (VRANKS + VPAD)];
    __shared__ int toks[16 * NT];
    const int m = mod_of(tab, blockIdx.x);
    const LoraMod& d = tab.mod[m];
    int at = blockIdx.x - tab.first[m];
    const int blocks = (int)((d.M + EXPAND_ROWS - 1) / EXPAND_ROWS), tile = at / blocks;
    const int64_t row0 = (int64_t)(at % blocks) * EXPAND_ROWS;
    int adapter, r;
    if (!find_tile<16 * NT>(c, tile, d.rank, toks, adapter, r)) return;
    if (r == 0 && d.y0 == d.y) return;         /* y already holds the result */
    const int lane = threadIdx.x % WAVE, wave = wsr::wave_in_block(), col = lane % 16, g = lane / 16;
    const float scale = adapter >= 0 && c.scales ? c.scales[adapter] : 1.f;
    const char* b = (const char*)d.b + (adapter < 0 ? 0 : adapter) * d.b_stride;
    const bool wide = d.rank % 4 == 0 && ((uintptr_t)b & 7) == 0;
    const int64_t i0 = row0 + wave * 64;
    f4_t acc[4][NT] = {};
    for (int j0 = 0; j0 < r; j0 += VRANKS) {
        const int q = (min(r - j0, VRANKS) + 15) / 16 * 4;     /* groups of four ranks of this round */
        if (j0) __syncthreads();
        for (int e = threadIdx.x; e < 16 * NT * q; e += LT) {
            const int tok = toks[e / q], j = e % q * 4;
            f4_t s = {0, 0, 0, 0};
            if (tok >= 0)
                for (int p = 0; p < d.parts; ++p)
                    s += *(const f4_t*)(d.v + ((int64_t)p * c.n_tokens + tok) * d.pitch + j0 + j);
            *(f4_t*)(vs + (e / q) * (VRANKS + VPAD) + j) = s * scale;
        }
        __syncthreads();
        for (int j = 0; j < 4 * q; j += 16) {
            const int jj = j + 4 * g;
            f4_t bv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t row = i0 + 16 * i + col;
                bv[i] = load_b4<FMT>(b + (row * d.rank + j0 + jj) * 2, row < d.M ? r - j0 - jj : 0, wide);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const f4_t vv = *(const f4_t*)(vs + (16 * t + col) * (VRANKS + VPAD) + jj);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[i][k], vv[k], acc[i][t], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int tok = toks[16 * t + col];
        if (tok < 0) continue;
        const float* src = d.y0 ? (const float*)((const char*)d.y0 + tok * d.y0_stride) : nullptr;
        float* dst = (float*)((char*)d.y + tok * d.y_stride);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t o = i0 + 16 * i + 4 * g;
            if (o + 4 <= d.M) {
                f4_t s = acc[i][t];
                if (src) s += *(const f4_any_t*)(src + o);
                *(f4_any_t*)(dst + o) = s;
            } else {
                for (int k = 0; o + k < d.M; ++k) dst[o + k] = acc[i][t][k] + (src ? src[o + k] : 0.f);
            }
        }
    }
}

/* Tokens in order of their adapters (those without one last) and the tiles of `cols` tokens.  The order
   inside an adapter follows from the atomics and may differ from run to run; a token's results do not
   depend on its place in a tile. */
__global__ __launch_bounds__(SORT_THREADS) void k_lora_sort(const int32_t* adapter_of, int n_tokens, int n_adapters,
                                                            int cols, int32_t* tiles, int32_t* order) {
    extern __shared__ int32_t bin[];           /* [n_adapters + 1] */
    __shared__ int32_t sc[SORT_THREADS], st[SORT_THREADS];
    const int n = n_adapters + 1, tid = threadIdx.x;
    for (int i = tid; i < n; i += SORT_THREADS) bin[i] = 0;
    __syncthreads();
    for (int t = tid; t < n_tokens; t += SORT_THREADS) {
        const int id = adapter_of[t];
        atomicAdd(&bin[id >= 0 && id < n_adapters ? id : n_adapters], 1);
    }
    __syncthreads();
    const int per = (n + SORT_THREADS - 1) / SORT_THREADS, b0 = min(n, tid * per), b1 = min(n, b0 + per);
    int tokens = 0, made = 0;
    for (int i = b0; i < b1; ++i) tokens += bin[i], made += (bin[i] + cols - 1) / cols;
    sc[tid] = tokens, st[tid] = made;
    __syncthreads();
    for (int k = 1; k < SORT_THREADS; k <<= 1) {
        const int a = tid >= k ? sc[tid - k] : 0, b = tid >= k ? st[tid - k] : 0;
        __syncthreads();
        sc[tid] += a, st[tid] += b;
        __syncthreads();
    }
    if (tid == SORT_THREADS - 1) tiles[0] = st[tid];
    int at = sc[tid] - tokens, tile = st[tid] - made;
    for (int i = b0; i < b1; ++i) {
        const int count = bin[i];
        for (int k = 0; k < count; k += cols, ++tile) {
            tiles[1 + 3 * tile] = i == n_adapters ? -1 : i;
            tiles[2 + 3 * tile] = at + k;
            tiles[3 + 3 * tile] = min(cols, count - k);
        }
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

static int tile_cols(int32_t n_tokens) { return n_tokens <= BALLOT_TOKENS ? 16 : 64; }
static int64_t most_tiles(int32_t n_tokens, int32_t n_adapters) {
    if (n_tokens <= BALLOT_TOKENS) return n_tokens;
    return n_tokens / tile_cols(n_tokens) + std::min<int64_t>(n_tokens, (int64_t)n_adapters + 1);
}

/* Parts of K of each projection: enough workgroups to fill the chip where the call is small, none under
   512 elements. */
static void part_of(const wsr_lora& m, int32_t n, int32_t n_tokens, int& parts, int& part_k) {
    const int64_t tiles = std::max<int64_t>(1, n_tokens / tile_cols(n_tokens));
    const int64_t want = std::max<int64_t>(1, 512 / (tiles * n)), most = std::max<int64_t>(1, (m.K + 511) / 512);
    const int64_t k = (m.K + std::min(want, most) - 1) / std::min(want, most);
    part_k = (int)std::max<int64_t>(32, (k + 31) / 32 * 32);
    parts = (int)std::max<int64_t>(1, (m.K + part_k - 1) / part_k);
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }
static size_t lists_bytes(int32_t n_tokens) {
    return n_tokens <= BALLOT_TOKENS ? 0 : up256(4 * (1 + 3 * (size_t)most_tiles(n_tokens, MAX_ADAPTERS))) + up256(4 * (size_t)n_tokens);
}

size_t lora_workspace(const wsr_lora* mods, int32_t n, int32_t n_tokens) {
    size_t bytes = lists_bytes(n_tokens);
    for (int32_t i = 0; i < n; ++i) {
        int parts, part_k;
        part_of(mods[i], n, n_tokens, parts, part_k);
        bytes += up256((size_t)parts * n_tokens * ((mods[i].rank + 15) / 16 * 16) * 4);
    }
    return std::max<size_t>(bytes, 256);
}

template <int FMT, int NT, int N>
static hipError_t launch_pair(const LoraTable<N>& tab0, const LoraCall& c, hipStream_t s) {
    LoraTable<N> tab = tab0;
    int64_t blocks = 0;
    for (int i = 0; i < tab.n; ++i) {
        tab.first[i] = (int32_t)blocks;
        blocks += (int64_t)tab.mod[i].parts * ((tab.mod[i].rank + RANKS - 1) / RANKS) * c.tile_slots;
    }
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_lora_shrink<FMT, NT, N>), dim3((unsigned)blocks), dim3(LT), 0, s, tab, c);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    blocks = 0;
    for (int i = 0; i < tab.n; ++i) {
        tab.first[i] = (int32_t)blocks;
        blocks += (tab.mod[i].M + EXPAND_ROWS - 1) / EXPAND_ROWS * c.tile_slots;
    }
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_lora_expand<FMT, NT, N>), dim3((unsigned)blocks), dim3(LT), 0, s, tab, c);
    return hipGetLastError();
}

template <int N>
static hipError_t launch_table(const LoraMod* mods, int n, int fmt, const LoraCall& c, hipStream_t s) {
    LoraTable<N> tab;
    tab.n = n;
    std::copy(mods, mods + n, tab.mod);
    const bool one = !c.tiles;
    if (fmt == WSR_F16) return one ? launch_pair<WSR_F16, 1, N>(tab, c, s) : launch_pair<WSR_F16, 4, N>(tab, c, s);
    return one ? launch_pair<WSR_BF16, 1, N>(tab, c, s) : launch_pair<WSR_BF16, 4, N>(tab, c, s);
}

constexpr int TABLE_MAX = 224;

hipError_t launch_lora(const wsr_lora* mods, int32_t n, int32_t n_tokens, const int32_t* adapter_of, int32_t n_adapters,
                       const int32_t* ranks, const float* scales, void* ws, hipStream_t s) {
    char* at = static_cast<char*>(ws);
    LoraCall c{};
    c.adapter_of = adapter_of, c.ranks = ranks, c.scales = scales, c.n_tokens = n_tokens, c.n_adapters = n_adapters;
    c.tile_slots = (int32_t)most_tiles(n_tokens, n_adapters);
    if (n_tokens > BALLOT_TOKENS) {
        int32_t* tiles = reinterpret_cast<int32_t*>(at);
        int32_t* order = reinterpret_cast<int32_t*>(at + up256(4 * (1 + 3 * (size_t)most_tiles(n_tokens, MAX_ADAPTERS))));
        at += lists_bytes(n_tokens);
        c.tiles = tiles, c.order = order;
        hipLaunchKernelGGL(k_lora_sort, dim3(1), dim3(SORT_THREADS), 4 * ((size_t)n_adapters + 1), s, adapter_of, n_tokens,
                           n_adapters, tile_cols(n_tokens), tiles, order);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    /* runs of projections of one type, at most a table's length */
    LoraMod run[TABLE_MAX];
    int held = 0;
    for (int32_t i = 0; i < n; ++i) {
        const wsr_lora& m = mods[i];
        LoraMod d{m.a, m.b, m.x, m.y0, m.y, reinterpret_cast<float*>(at), m.a_stride, m.b_stride, m.x_tok_stride,
                  m.y0_tok_stride, m.y_tok_stride, m.M, m.K, m.rank, (m.rank + 15) / 16 * 16, 1, 0};
        part_of(m, n, n_tokens, d.parts, d.part_k);
        at += up256((size_t)d.parts * n_tokens * d.pitch * 4);
        run[held++] = d;
        if (held == TABLE_MAX || i + 1 == n || mods[i + 1].fmt != m.fmt) {
            const hipError_t e = held <= 8 ? launch_table<8>(run, held, m.fmt, c, s)
                                           : launch_table<TABLE_MAX>(run, held, m.fmt, c, s);
            if (e != hipSuccess) return e;
            held = 0;
        }
    }
    return hipSuccess;
}

}  // namespace wsr_step
