// Products with many rows a group: tiles of up to 256 rows of x against 256 rows of the weights, one workgroup of four
// waves (2 x 2 over the tile) per CU.
//
// Both operands go from memory straight into LDS (loads that write LDS, ffn_common.h) in slabs of 128 bytes a row, whole
// lines: a CU gets 123 GB/s that way, and 38 where lanes load operand fragments of row-major weights themselves (16 rows a
// request; the same tile 265 us so, 8192 x 4096 x 7168).  An LDS row is unpadded, its eight 16-byte pieces in the order piece ^
// (row & 7), so that the reads of a fragment hit every bank once.  A slab is two steps of 64 bytes.  While one step is multiplied,
// all fragments of the next are read into the other set of registers: behind the first step of a slab its stage
// is free again, and the slab that takes its place is requested at once.  Every memory instruction is dealt out behind a matrix
// instruction of its own.
//
// Groups are cut into full tiles of `height` rows and one remainder: of more than 64 rows a lower tile, of fewer units
// of product_stream.h.  The list has all full tiles first, then remainders.
#pragma once

#include <algorithm>
#include <type_traits>

#include "ffn_common.h"
#include "product_stream.h"

namespace craft {
namespace {

constexpr int kThreads = 256;
constexpr int kTileColumns = 256;                  // weight rows of a tile (gated: half of them gate, half up)
constexpr int kSlab = 128;                         // bytes of the contraction
constexpr int kTileLds = 2 * 512 * kSlab;
template <int FW, int FX> constexpr int tile_stages() { return 3 * (FW + FX) * 32 * kSlab <= kTileLds + (16 << 10) ? 3 : 2; }
template <bool GATED> constexpr int unit_columns() { return GATED ? 16 : 32; }        // of a remainder's unit
static_assert(kStreamWaves * 64 == kThreads && kStreamWaves * kRingBytes <= kTileLds + (16 << 10), "units in a tile's LDS");

template <int FMT> static __device__ __forceinline__ void multiply_in_place(raw_t w, raw_t x, typename Numbers<FMT>::acc_t &c) {
    if constexpr (FMT == CRAFT_I8) {
        asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
    } else if constexpr (FMT == CRAFT_BF16) {
        asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t p = w[e], q = x[e];
            asm("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
        }
    }
}

struct Tile {
    int32_t group, rows, n0;       // n0: first column of the result
    int64_t row0;
};

// FW, FX: 16-row fragments of weights and of x per wave; the tile is 32 FW columns (gated: 16 FW) x 32 FX rows.
template <int FMT, bool GATED, int FW, int FX>
static __device__ __forceinline__ void product_tile(const ProductArgs &a, const Tile &t, unsigned char *smem, float *row_scale, uint8_t *row_live) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int M = FW * FX, NR = FW + FX, STAGE = NR * 32 * kSlab, S = tile_stages<FW, FX>();
    static_assert(S * STAGE <= kTileLds + (16 << 10), "stages");
    const int lane = threadIdx.x & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t KB = a.row_bytes, nk = (KB + kSlab - 1) / kSlab;
    // Chunk 4 i + wave, eight rows of an operand, is this wave's i-th.  In front of LDS: weights, then x.
    const uint32_t piece = (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7)) * 16);
    const bool gather = a.src != nullptr;
    const ubase_t xbase = uniform_base(gather ? a.x : a.x + t.row0 * a.x_stride);
    uint32_t woff[FW], xoff[FX];
#pragma unroll
    for (int i = 0; i < FX; ++i) {
        const int r = min(8 * (4 * i + wave) + (lane >> 3), t.rows - 1);
        const int64_t tok = gather ? token_of(a, t.row0 + r) : r;
        xoff[i] = (uint32_t)((tok < 0 ? 0 : tok) * a.x_stride) + piece;
    }
    if ((int)threadIdx.x < t.rows) {
        const int64_t tok = token_of(a, t.row0 + threadIdx.x);
        row_live[threadIdx.x] = tok >= 0;
        if (FMT == CRAFT_I8) row_scale[threadIdx.x] = a.x_scale[tok < 0 ? 0 : tok];
    }
    // Gated: 16 rows of gate are followed by the 16 of up of the same columns; the first two waves fetch gate's.
    const unsigned char *mat = a.off ? a.w[t.group] : a.w_one;
    if (GATED && wave >= 2) mat = a.up[t.group];
    const ubase_t wbase = uniform_base(mat + (int64_t)t.n0 * KB);
    auto column = [](int r) { return GATED ? (r >> 5) * 16 + (r & 15) : r; };
#pragma unroll
    for (int i = 0; i < FW; ++i) woff[i] = (uint32_t)min(column(8 * (4 * i + wave) + (lane >> 3)), a.N - 1 - t.n0) * (uint32_t)KB + piece;

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane(wave * 1024);
    const uint32_t fo = lds0 + (uint32_t)(r16 * 128 + ((q ^ (lane & 7)) & 7) * 16);
    const uint32_t fw0 = fo + (uint32_t)((wave >> 1) * FW * 2048), fx0 = fo + (uint32_t)((2 * FW + (wave & 1) * FX) * 2048);
    typedef const raw_t __attribute__((address_space(3))) *frag_t;

    raw_t wv[2][FW], xv[2][FX];
    acc_t acc[FW][FX];
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int g = 0; g < FX; ++g) acc[f][g] = acc_t{};

    // where slab ks begins in a row: the last one ends with it, and what the one before has is cut away
    auto at = [&](int ks) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane(min(ks * kSlab, KB - kSlab)); };
    auto aim = [&](int i, uint32_t stage) __attribute__((always_inline)) { dma_to(lds_wave + stage + (uint32_t)(4096 * i)); };
    auto request = [&](int i, uint32_t k) __attribute__((always_inline)) {
        if (i < FW) dma_request(wbase + k, woff[i < FW ? i : 0]);
        else dma_request(xbase + k, xoff[i < FW ? 0 : i - FW]);
    };
    // x's fragments first, the next products start with those
    struct From { uint32_t x, w; };                // one register each, fragments at constant offsets from them
    auto from = [&](int step, uint32_t stage) __attribute__((always_inline)) {
        From p = {(fx0 ^ (step ? 64u : 0u)) + stage, (fw0 ^ (step ? 64u : 0u)) + stage};
        asm volatile("" : "+v"(p.x), "+v"(p.w));
        return p;
    };
    auto fetch = [&](int set, int j, const From &p) __attribute__((always_inline)) {
        if (j < FX) xv[set][j < FX ? j : 0] = *(frag_t)(uintptr_t)(p.x + (uint32_t)(j * 2048));
        else wv[set][j < FX ? 0 : j - FX] = *(frag_t)(uintptr_t)(p.w + (uint32_t)((j - FX) * 2048));
    };
    // bytes of the last slab that the one before it has already; a matrix instruction may read what a vector instruction wrote
    // two cycles later
    auto cut = [&](int set) __attribute__((always_inline)) {
        const bool gone = set * 64 + q * 16 < nk * kSlab - KB;
#pragma unroll
        for (int g = 0; g < FX; ++g) {
            xv[set][g] = gone ? raw_t{} : xv[set][g];
            asm volatile("s_nop 1" : "+v"(xv[set][g]));
        }
#pragma unroll
        for (int f = 0; f < FW; ++f) {
            wv[set][f] = gone ? raw_t{} : wv[set][f];
            asm volatile("s_nop 1" : "+v"(wv[set][f]));
        }
    };
    // One step: set STEP multiplied, the other one read from `stage`; DMA: slab `k` requested into `to` as well.
    auto step_of = [&](auto STEP, auto DMA, uint32_t stage, uint32_t to, uint32_t k) __attribute__((always_inline)) {
        constexpr int set = STEP.value, OPS = DMA.value ? 3 * NR : NR;
        const From p = from(set ^ 1, stage);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            multiply_in_place<FMT>(wv[set][m / FX], xv[set][m % FX], acc[m / FX][m % FX]);
            // spread over three quarters of the step: what is read has to be there when the next one begins
#pragma unroll
            for (int o = min(m * OPS * 4 / (3 * M), OPS); o < min((m + 1) * OPS * 4 / (3 * M), OPS); ++o) {
                if (!DMA.value) {
                    fetch(set ^ 1, o, p);
                } else if (o % 3 == 0) {
                    dma_to(lds_wave + to + (uint32_t)(4096 * (o / 3)));
                } else if (o % 3 == 1) {
                    fetch(set ^ 1, o / 3, p);
                } else {
                    request(o / 3, k);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const std::integral_constant<int, 0> step0;
    const std::integral_constant<int, 1> step1;
    const std::true_type with;
    const std::false_type without;
    const bool cuts = nk * kSlab != KB;

#pragma unroll
    for (int j = 0; j < S; ++j)
        if (j < nk) {
            const uint32_t k = at(j);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                aim(i, j * STAGE);
                asm volatile("s_nop 0");
                request(i, k);
            }
        }
    if (nk >= S) dma_wait<(S - 1) * NR>();
    else dma_wait<0>();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NR; ++j) fetch(0, j, from(0, 0));
    uint32_t here = 0;
    int ks = 0;
    // Behind the first step all of slab ks is in registers, for every wave at the barrier, and slab ks + 1 has landed: what is
    // on its way by then are the slabs behind it.
    for (; ks + S < nk; ++ks) {
        const uint32_t there = here + STAGE < S * STAGE ? here + STAGE : 0;
        step_of(step0, without, here, 0, 0);
        dma_wait<(S - 2) * NR>();
        __syncthreads();
        step_of(step1, with, there, here, at(ks + S));
        here = there;
    }
    for (; ks < nk; ++ks) {
        const uint32_t there = here + STAGE < S * STAGE ? here + STAGE : 0;
        const bool last = ks + 1 == nk;
        if (last && cuts) cut(0);
        step_of(step0, without, here, 0, 0);
        dma_wait<0>();
        __syncthreads();
        if (last && cuts) cut(1);
        step_of(step1, without, there, 0, 0);      // (behind the last slab: read and not used)
        here = there;
    }
    // a matrix instruction's result is read: idle cycles, then every accumulator through a statement behind them
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int g = 0; g < FX; ++g) asm volatile("" : "+a"(acc[f][g]));

    // element v of lane l is column 4 (l >> 4) + v and row l & 15 of its fragment
    constexpr int SIDES = GATED ? 2 : 1;
    const int32_t col0 = t.n0 + column((wave >> 1) * FW * 16) + 4 * q;
    float ws[FW][4];
    if (FMT == CRAFT_I8) {
        const scales_t s0 = (scales_t)(a.off ? a.w_scale[t.group] : a.w_one_scale), s1 = GATED ? (scales_t)a.up_scale[t.group] : s0;
#pragma unroll
        for (int f = 0; f < FW; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t c = min(col0 + f / SIDES * 16 + e, a.N - 1);
                if (f & (SIDES - 1)) ws[f][e] = s1[c];
                else ws[f][e] = s0[c];
            }
    }
    // By way of LDS, 16 rows at a time and each wave for itself, so that a store covers whole lines (16 rows of 32 bytes a
    // request: 8 us a tile where this takes 3).  Stores are of 16 bytes whatever the alignment; a lane at the matrix' edge
    // stores its columns one by one.
    auto results = [&](auto BF16) __attribute__((always_inline)) {
        constexpr bool bf16 = BF16.value;
        typedef typename std::conditional<bf16, uint16_t, float>::type out_t;
        typedef out_t piece_t __attribute__((ext_vector_type(16 / sizeof(out_t)), aligned(sizeof(out_t))));
        constexpr int COLS = 16 * FW / SIDES, ROWB = COLS * (int)sizeof(out_t), PITCH = ROWB + 16;     // a row of this wave
        constexpr int PER = ROWB / 16, EACH = 16 / (int)sizeof(out_t), PASSES = 16 * PER / 64;      // pieces of a row; elements of a piece
        static_assert(4 * 16 * PITCH <= kTileLds, "rows of results");
        unsigned char *const mine = smem + wave * (16 * PITCH);
        const int32_t first = t.n0 + (wave >> 1) * COLS;
        out_t *const out = static_cast<out_t *>(a.out) + first;
#pragma unroll
        for (int g = 0; g < FX; ++g) {
            int l = lane;                          // (places are worked out here, not in front of the loop for all of it)
            asm volatile("" : "+v"(l));
            const int row = (wave & 1) * FX * 16 + 16 * g + (l & 15);
            const float xs = FMT == CRAFT_I8 ? row_scale[row] : 1.0f;
            const bool live = row_live[row];
#pragma unroll
            for (int f = 0; f < FW; f += SIDES) {
                float v[SIDES][4];
#pragma unroll
                for (int m = 0; m < SIDES; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[m][e] = FMT == CRAFT_I8 ? (float)acc[f + m][g][e] * xs * ws[f + m][e] : (float)acc[f + m][g][e];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (GATED) v[0][e] = (bf16 ? silu_bf16(v[0][e]) : silu_f32(v[0][e])) * v[SIDES - 1][e];
                    v[0][e] = live ? v[0][e] : 0.0f;
                }
                unsigned char *p = mine + (l & 15) * PITCH + (f / SIDES * 16 + 4 * (l >> 4)) * (int)sizeof(out_t);
                if constexpr (bf16) *reinterpret_cast<uint2 *>(p) = make_uint2(product_bf16_pair(v[0][0], v[0][1]), product_bf16_pair(v[0][2], v[0][3]));
                else *reinterpret_cast<float4 *>(p) = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
            }
            // (the wave's own rows: its reads follow its writes)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = (i * 64 + l) / PER, c = (i * 64 + l) % PER * EACH, at = (wave & 1) * FX * 16 + 16 * g + r;
                const unsigned char *from = mine + r * PITCH + c * (int)sizeof(out_t);
                const raw_t v = *reinterpret_cast<const raw_t *>(from);
                if (at < t.rows) {
                    out_t *p = out + (t.row0 + at) * a.out_stride + c;
                    if (first + c + EACH <= a.N) *reinterpret_cast<piece_t *>(p) = __builtin_bit_cast(piece_t, v);
                    else
#pragma unroll 1
                        for (int e = 0; first + c + e < a.N; ++e) p[e] = reinterpret_cast<const out_t *>(from)[e];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    __syncthreads();                               // every wave has read the last slab
    if (FMT != CRAFT_F32 && a.out_dtype == CRAFT_BF16) results(with);
    else results(without);
    __syncthreads();                               // LDS may be filled again
}

// How many full tiles, remaining tiles and remaining units the groups in front of one have: [G + 1] each, in LDS.
struct Counts {
    int32_t full[kMostGroups + 1], low[kMostGroups + 1], few[kMostGroups + 1];
};
static __device__ __forceinline__ void count_tiles(const ProductArgs &a, int32_t height, Counts &n, int32_t *scratch) {
    if (!a.off) {                                  // one group
        if (threadIdx.x == 0) {
            const int32_t rest = (int32_t)(a.M % height);
            n.full[0] = n.low[0] = n.few[0] = 0;
            n.full[1] = (int32_t)(a.M / height);
            n.low[1] = rest > kUnitRows;
            n.few[1] = rest > 0 && rest <= kUnitRows;
        }
        __syncthreads();
        return;
    }
    const int32_t each = (a.G + kThreads - 1) / kThreads, first = min((int32_t)threadIdx.x * each, a.G), last = min(first + each, a.G);
    int32_t sum[3] = {0, 0, 0};
    for (int32_t g = first; g < last; ++g) {
        int64_t lo, hi;
        group_rows(a, g, lo, hi);
        const int32_t rows = (int32_t)(hi - lo), rest = rows % height;
        n.full[g] = rows / height;
        n.low[g] = rest > kUnitRows;
        n.few[g] = rest > 0 && rest <= kUnitRows;
        sum[0] += n.full[g];
        sum[1] += n.low[g];
        sum[2] += n.few[g];
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) scratch[i * kThreads + threadIdx.x] = sum[i];
    __syncthreads();
    for (int d = 1; d < kThreads; d *= 2) {
        int32_t add[3] = {0, 0, 0};
        if ((int)threadIdx.x >= d)
#pragma unroll
            for (int i = 0; i < 3; ++i) add[i] = scratch[i * kThreads + threadIdx.x - d];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 3; ++i) scratch[i * kThreads + threadIdx.x] += add[i];
        __syncthreads();
    }
    int32_t *const out[3] = {n.full, n.low, n.few};
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        int32_t at = scratch[i * kThreads + threadIdx.x] - sum[i];
        for (int32_t g = first; g < last; ++g) {
            const int32_t c = out[i][g];
            out[i][g] = at;
            at += c;
        }
        if (threadIdx.x == kThreads - 1) out[i][a.G] = scratch[i * kThreads + kThreads - 1];
    }
    __syncthreads();
}
// before[g] <= i < before[g + 1]
static __device__ __forceinline__ int32_t group_of(const int32_t *before, int32_t G, int32_t i) {
    int32_t lo = 0, hi = G;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (before[mid] <= i) lo = mid; else hi = mid;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Item i of a group's m x nt tiles: blocks of 8 x 8, column by column inside a block, so that the tiles that run at one
// time need few rows of either operand between them.
static __device__ __forceinline__ void place(int32_t i, int32_t m, int32_t nt, int32_t &row, int32_t &col) {
    const int32_t band = i / (8 * nt), r0 = band * 8, rj = min(8, m - r0), in = i - r0 * nt;
    const int32_t block = in / (rj * 8), rest = in - block * rj * 8;
    row = r0 + rest % rj;
    col = block * 8 + rest / rj;
}

template <int FMT, bool GATED>
__global__ __launch_bounds__(kThreads, 1) void product_tile_kernel(ProductArgs a, int32_t height) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[kTileLds + (16 << 10)];
    __shared__ Counts n;
    __shared__ float row_scale[256];
    __shared__ uint8_t row_live[256];
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int COLS = GATED ? kTileColumns / 2 : kTileColumns, REM = unit_columns<GATED>() / 16;
    count_tiles(a, height, n, reinterpret_cast<int32_t *>(smem));
    const int32_t nt = (a.N + COLS - 1) / COLS, nu = (a.N + 16 * REM - 1) / (16 * REM);
    const int64_t full = (int64_t)n.full[a.G] * nt, low = full + (int64_t)n.low[a.G] * nt, all = low + (int64_t)n.few[a.G] * nu;
    int64_t w = blockIdx.x;
    {
        // neighbours in the list start together on one XCD
        const int64_t run = gridDim.x / 8;
        w = (w % 8) * run + w / 8;
    }
    for (; w < low; w += gridDim.x) {
        Tile t;
        int64_t lo, hi;
        int32_t tr, tc;
        const bool is_full = w < full;
        const int32_t *before = is_full ? n.full : n.low;
        const int64_t i = is_full ? w : w - full;
        t.group = group_of(before, a.G, (int32_t)(i / nt));
        group_rows(a, t.group, lo, hi);
        if (is_full) {
            place((int32_t)(i - (int64_t)before[t.group] * nt), before[t.group + 1] - before[t.group], nt, tr, tc);
            t.rows = height;
        } else {
            tr = (int32_t)((hi - lo) / height);
            tc = (int32_t)(i % nt);
            t.rows = (int32_t)(hi - lo) - tr * height;
        }
        t.row0 = lo + (int64_t)tr * height;
        t.n0 = tc * COLS;
        t.rows = __builtin_amdgcn_readfirstlane(t.rows);
        t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
        if (t.rows <= 64) product_tile<FMT, GATED, 8, 2>(a, t, smem, row_scale, row_live);
        else if (t.rows <= 128) product_tile<FMT, GATED, 8, 4>(a, t, smem, row_scale, row_live);
        else if (t.rows <= 192) product_tile<FMT, GATED, 8, 6>(a, t, smem, row_scale, row_live);
        else product_tile<FMT, GATED, 8, 8>(a, t, smem, row_scale, row_live);
    }
    for (; w < all; w += gridDim.x) {
        const int64_t i = w - low;
        Unit u;
        int64_t lo, hi;
        u.group = group_of(n.few, a.G, (int32_t)(i / nu));
        group_rows(a, u.group, lo, hi);
        u.n0 = __builtin_amdgcn_readfirstlane((int32_t)(i % nu) * 16 * REM);
        u.rows = __builtin_amdgcn_readfirstlane((int32_t)((hi - lo) % height));
        u.row0 = hi - u.rows;
        acc_t *part = reinterpret_cast<acc_t *>(smem);
        unsigned char *const ring = smem + ((int)threadIdx.x >> 6) * kRingBytes;
        if (u.rows <= 16) stream_unit<FMT, GATED, REM, 1, kStreamWaves>(a, u, ring, part);
        else if (u.rows <= 32) stream_unit<FMT, GATED, REM, 2, kStreamWaves>(a, u, ring, part);
        else stream_unit<FMT, GATED, REM, 4, kStreamWaves>(a, u, ring, part);
    }
}

template <int FMT> hipError_t launch_tiles(const ProductArgs &a, int32_t height, hipStream_t s) {
    const int cols = a.up ? kTileColumns / 2 : kTileColumns;
    const int64_t nt = (a.N + cols - 1) / cols, nu = (a.N + 15) / 16;
    const int64_t bound = (a.M / height) * nt + std::min<int64_t>(a.M, a.G) * nu;
    const int64_t grid = std::max<int64_t>(8, (std::min<int64_t>(bound, a.num_cu) + 7) / 8 * 8);
    if (a.up) hipLaunchKernelGGL((product_tile_kernel<FMT, true>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, height);
    else hipLaunchKernelGGL((product_tile_kernel<FMT, false>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, height);
    return hipGetLastError();
}

}  // namespace
}  // namespace craft
