// Products with many rows a group: tiles of up to 256 rows of x against 256 rows of the weights, one workgroup of four
// waves per CU.
//
// Rows of x go from memory straight into LDS (loads that write LDS, ffn_common.h), in slabs of 128 bytes, four
// stages, three slabs ahead; every wave reads all of them as operand fragments.  Each wave has 64 weight rows of its own,
// whose fragments it loads straight into registers, four slabs ahead: nobody else needs them, and LDS then carries 80
// bytes a cycle at full speed where both operands by way of it would be 96 (of 128).  A step of 64 bytes is multiplied in
// halves of the tile's rows, while one half is multiplied the other's fragments are fetched; every memory instruction
// is dealt out behind a matrix instruction of its own.
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
constexpr int kStages = 4;
constexpr int kSlab = 128;                         // bytes of the contraction
constexpr int kStageBytes = 256 * kSlab;
constexpr int kRemCF = 2;                          // columns / 16 of a remainder's unit

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

// 32 HF rows against four waves' 16 CF weight rows each.
template <int FMT, bool GATED, int HF, int CF>
static __device__ __forceinline__ void product_tile(const ProductArgs &a, const Tile &t, unsigned char *smem, float *row_scale, uint8_t *row_live) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int M = HF * CF;
    const int lane = threadIdx.x & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t KB = a.row_bytes, nk = (KB + kSlab - 1) / kSlab;
    // Rows of x: chunk 4 i + wave of eight rows is this wave's i-th.
    const bool gather = a.src != nullptr;
    const ubase_t xbase = uniform_base(gather ? a.x : a.x + t.row0 * a.x_stride);
    uint32_t aoff[HF];
#pragma unroll
    for (int i = 0; i < HF; ++i) {
        const int r = min(8 * (4 * i + wave) + (lane >> 3), t.rows - 1);
        const int64_t tok = gather ? token_of(a, t.row0 + r) : r;
        aoff[i] = (uint32_t)((tok < 0 ? 0 : tok) * a.x_stride) + (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7)) * 16);
    }
    if ((int)threadIdx.x < t.rows) {
        const int64_t tok = token_of(a, t.row0 + threadIdx.x);
        row_live[threadIdx.x] = tok >= 0;
        if (FMT == CRAFT_I8) row_scale[threadIdx.x] = a.x_scale[tok < 0 ? 0 : tok];
    }
    // Weight rows: fragment c of this wave is 16 columns (gated: of gate and up in turn).
    const ubase_t w0 = uniform_base(a.off ? a.w[t.group] : a.w_one), w1 = GATED ? uniform_base(a.up[t.group]) : w0;
    constexpr int SIDES = GATED ? 2 : 1;
    auto column = [&](int c) { return t.n0 + (wave * (CF / SIDES) + c / SIDES) * 16; };
    uint32_t boff[CF];
    const ubase_t wt0 = w0 + (int64_t)t.n0 * KB, wt1 = w1 + (int64_t)t.n0 * KB;
#pragma unroll
    for (int c = 0; c < CF; ++c) boff[c] = (uint32_t)(min(column(c) + r16, a.N - 1) - t.n0) * (uint32_t)KB + (uint32_t)(q * 16);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane(wave * 1024);
    const uint32_t fo = lds0 + (uint32_t)(r16 * 128 + ((q ^ (lane & 7)) & 7) * 16);
    typedef const raw_t __attribute__((address_space(3))) *frag_t;

    raw_t av[2][HF], bv[4][2][CF];
    acc_t acc[2 * HF][CF];
#pragma unroll
    for (int f = 0; f < 2 * HF; ++f)
#pragma unroll
        for (int c = 0; c < CF; ++c) acc[f][c] = acc_t{};

    // where slab ks begins in a row: the last one ends with it, and what the one before has is cut away
    auto at = [&](int ks) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane(min(ks * kSlab, KB - kSlab)); };
    auto aim = [&](int i, int stage) __attribute__((always_inline)) { dma_to(lds_wave + (uint32_t)(stage * kStageBytes + 4096 * i)); };
    auto request = [&](int i, uint32_t k) __attribute__((always_inline)) { dma_request(xbase + k, aoff[i]); };
    auto weights = [&](int u, int step, int c, uint32_t k) __attribute__((always_inline)) {
        bv[u][step][c] = wload<false, raw_t>(((c & (SIDES - 1)) ? wt1 : wt0) + k + step * 64, boff[c]);
    };
    auto fetch = [&](int half, int stage, int f) __attribute__((always_inline)) {
        const uint32_t base = (half & 2 ? fo ^ 64u : fo) + (uint32_t)(stage * kStageBytes);
        av[half & 1][f] = *(frag_t)(uintptr_t)(base + (uint32_t)(((half & 1) * HF + f) * 2048));
    };
    auto cut_a = [&](int half) __attribute__((always_inline)) {
        const bool gone = (half & 2 ? 64 : 0) + q * 16 < nk * kSlab - KB;
#pragma unroll
        for (int f = 0; f < HF; ++f) {
            av[half & 1][f] = gone ? raw_t{} : av[half & 1][f];
            asm volatile("s_nop 1" : "+v"(av[half & 1][f]));
        }
    };
    auto cut_b = [&](int u) __attribute__((always_inline)) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const bool gone = step * 64 + q * 16 < nk * kSlab - KB;
#pragma unroll
            for (int c = 0; c < CF; ++c) {
                bv[u][step][c] = gone ? raw_t{} : bv[u][step][c];
                asm volatile("s_nop 1" : "+v"(bv[u][step][c]));
            }
        }
    };
    // Half `half` of the slab in stage u: columns outside, so that a column's weights are free behind its products.
    // dma: rows of slab ks + 3 are requested (in halves 0 and 1); more: weights of slab ks + 4 (in half 3).
    auto half_of = [&](auto U, auto HALF, bool dma, bool more, uint32_t kdma, uint32_t kmore) __attribute__((always_inline)) {
        constexpr int u = U.value, half = HALF.value, next = (half + 1) & 3, next_stage = half == 3 ? (u + 1) & 3 : u;
        constexpr int D0 = half == 0 ? 0 : (HF + 1) / 2, ND = half == 0 ? (HF + 1) / 2 : half == 1 ? HF / 2 : 0;
        constexpr int OPS = HF + 2 * ND;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int c = m / HF, f = m % HF;
            multiply_in_place<FMT>(bv[u][half >> 1][c], av[half & 1][f], acc[(half & 1) * HF + f][c]);
#pragma unroll
            for (int o = m * OPS / M; o < (m + 1) * OPS / M; ++o) {
                if (o < HF) fetch(next, next_stage, o);
                else if (dma) {
                    const int i = D0 + (o - HF) / 2;
                    if ((o - HF) % 2 == 0) aim(i, (u + 3) & 3);
                    else {
                        if (o > m * OPS / M) asm volatile("s_nop 0");
                        request(i, kdma);
                    }
                }
            }
            if (half == 3 && f == HF - 1 && more) {
                weights(u, 0, c, kmore);
                weights(u, 1, c, kmore);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const bool cuts = nk * kSlab != KB;
    // AHEAD: everything that is requested exists
    auto slab = [&](auto U, auto AHEAD, int ks) __attribute__((always_inline)) {
        constexpr int u = U.value;
        constexpr bool ahead = AHEAD.value;
        const bool dma = ahead || ks + 3 < nk, more = ahead || ks + 4 < nk, last = !ahead && ks + 1 == nk;
        const uint32_t kdma = at(ks + 3), kmore = at(ks + 4);
        if (last && cuts) { cut_b(u); cut_a(0); }
        half_of(U, std::integral_constant<int, 0>{}, dma, more, kdma, kmore);
        if (last && cuts) cut_a(1);
        half_of(U, std::integral_constant<int, 1>{}, dma, more, kdma, kmore);
        if (last && cuts) cut_a(2);
        half_of(U, std::integral_constant<int, 2>{}, dma, more, kdma, kmore);
        // Slab ks + 1 has landed when at most what was requested behind it is on its way: weights and rows of two slabs
        // (the tail: fewer).  At the barrier all of slab ks has been read by every wave.
        if (dma) dma_wait<4 * CF + 2 * HF>();
        else if (ks + 3 == nk) dma_wait<2 * CF + HF>();
        else dma_wait<0>();
        __syncthreads();
        if (last && cuts) cut_a(3);
        half_of(U, std::integral_constant<int, 3>{}, dma, more, kdma, kmore);
    };
    const std::integral_constant<int, 0> u0;
    const std::integral_constant<int, 1> u1;
    const std::integral_constant<int, 2> u2;
    const std::integral_constant<int, 3> u3;

    auto start_rows = [&](int j) __attribute__((always_inline)) {
        if (j < nk) {
#pragma unroll
            for (int i = 0; i < HF; ++i) {
                aim(i, j);
                asm volatile("s_nop 0");
                request(i, at(j));
            }
        }
    };
    auto start_weights = [&](auto J) __attribute__((always_inline)) {
        constexpr int j = J.value;
        if (j < nk)
#pragma unroll
            for (int c = 0; c < CF; ++c) {
                weights(j, 0, c, at(j));
                weights(j, 1, c, at(j));
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    start_rows(0);
    start_weights(u0);
    start_rows(1);
    start_weights(u1);
    start_rows(2);
    start_weights(u2);
    start_weights(u3);
    if (nk > 3) dma_wait<8 * CF + 2 * HF <= 63 ? 8 * CF + 2 * HF : 63>();
    else dma_wait<0>();
    __syncthreads();
#pragma unroll
    for (int f = 0; f < HF; ++f) fetch(0, 0, f);
    int ks = 0;
    const std::true_type ahead;
    const std::false_type bounded;
    for (; ks + 8 <= nk; ks += 4) {
        slab(u0, ahead, ks);
        slab(u1, ahead, ks + 1);
        slab(u2, ahead, ks + 2);
        slab(u3, ahead, ks + 3);
    }
    for (; ks < nk; ks += 4) {
        slab(u0, bounded, ks);
        if (ks + 1 >= nk) break;
        slab(u1, bounded, ks + 1);
        if (ks + 2 >= nk) break;
        slab(u2, bounded, ks + 2);
        if (ks + 3 >= nk) break;
        slab(u3, bounded, ks + 3);
    }
    // a matrix instruction's result is read: idle cycles, then every accumulator through a statement behind them
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int f = 0; f < 2 * HF; ++f)
#pragma unroll
        for (int c = 0; c < CF; ++c) asm volatile("" : "+a"(acc[f][c]));

    // element v of lane l is column 4 (l >> 4) + v and row l & 15 of its fragment
    const bool accurate = FMT == CRAFT_F32 || a.out_dtype == CRAFT_F32;
    const float *scales[SIDES] = {};
    if (FMT == CRAFT_I8) {
        scales[0] = a.off ? a.w_scale[t.group] : a.w_one_scale;
        if (GATED) scales[SIDES - 1] = a.up_scale[t.group];
    }
    float ws[CF][4];
    if (FMT == CRAFT_I8)
#pragma unroll
        for (int c = 0; c < CF; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) ws[c][e] = scales[c & (SIDES - 1)][min(column(c) + 4 * q + e, a.N - 1)];
#pragma unroll
    for (int f = 0; f < 2 * HF; ++f) {
        const int row = 16 * f + r16;
        if (row < t.rows) {
            const float xs = FMT == CRAFT_I8 ? row_scale[row] : 1.0f;
            const bool live = row_live[row];
#pragma unroll
            for (int c = 0; c < CF; c += SIDES) {
                const int32_t col = column(c) + 4 * q;
                float v[SIDES][4];
#pragma unroll
                for (int m = 0; m < SIDES; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[m][e] = FMT == CRAFT_I8 ? (float)acc[f][c + m][e] * xs * ws[c + m][e] : (float)acc[f][c + m][e];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (GATED) v[0][e] = silu_of(v[0][e], accurate) * v[1][e];
                    v[0][e] = live ? v[0][e] : 0.0f;
                }
                if (col < a.N) store_columns(a, t.row0 + row, col, v[0], a.out_whole);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();                               // LDS may be filled again
}

// How many full tiles, remaining tiles and remaining units the groups in front of one have: [G + 1] each, in LDS.
struct Counts {
    int32_t full[kMostGroups + 1], low[kMostGroups + 1], few[kMostGroups + 1];
};
static __device__ __forceinline__ void count_tiles(const ProductArgs &a, int32_t height, Counts &n, int32_t *scratch) {
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
    __shared__ __attribute__((aligned(16))) unsigned char smem[kStages * kStageBytes];
    __shared__ Counts n;
    __shared__ float row_scale[256];
    __shared__ uint8_t row_live[256];
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int COLS = GATED ? kTileColumns / 2 : kTileColumns;
    count_tiles(a, height, n, reinterpret_cast<int32_t *>(smem));
    const int32_t nt = (a.N + COLS - 1) / COLS, nu = (a.N + 16 * kRemCF - 1) / (16 * kRemCF);
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
        if (t.rows <= 64) product_tile<FMT, GATED, 2, 4>(a, t, smem, row_scale, row_live);
        else if (t.rows <= 128) product_tile<FMT, GATED, 4, 4>(a, t, smem, row_scale, row_live);
        else if (t.rows <= 192) product_tile<FMT, GATED, 6, 4>(a, t, smem, row_scale, row_live);
        else product_tile<FMT, GATED, 8, 4>(a, t, smem, row_scale, row_live);
    }
    for (; w < all; w += gridDim.x) {
        const int64_t i = w - low;
        Unit u;
        int64_t lo, hi;
        u.group = group_of(n.few, a.G, (int32_t)(i / nu));
        group_rows(a, u.group, lo, hi);
        u.n0 = __builtin_amdgcn_readfirstlane((int32_t)(i % nu) * 16 * kRemCF);
        u.rows = __builtin_amdgcn_readfirstlane((int32_t)((hi - lo) % height));
        u.row0 = hi - u.rows;
        acc_t *part = reinterpret_cast<acc_t *>(smem);
        if (u.rows <= 16) stream_unit<FMT, GATED, kRemCF, 1, 4>(a, u, part);
        else if (u.rows <= 32) stream_unit<FMT, GATED, kRemCF, 2, 4>(a, u, part);
        else stream_unit<FMT, GATED, kRemCF, 4, 4>(a, u, part);
    }
}

template <int FMT> hipError_t launch_tiles(const ProductArgs &a, int32_t height, hipStream_t s) {
    const int cols = a.up ? kTileColumns / 2 : kTileColumns;
    const int64_t nt = (a.N + cols - 1) / cols, nu = (a.N + 16 * kRemCF - 1) / (16 * kRemCF);
    const int64_t bound = (a.M / height) * nt + std::min<int64_t>(a.M, a.G) * nu;
    const int64_t grid = std::max<int64_t>(8, (std::min<int64_t>(bound, a.num_cu) + 7) / 8 * 8);
    if (a.up) hipLaunchKernelGGL((product_tile_kernel<FMT, true>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, height);
    else hipLaunchKernelGGL((product_tile_kernel<FMT, false>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, height);
    return hipGetLastError();
}

}  // namespace
}  // namespace craft
