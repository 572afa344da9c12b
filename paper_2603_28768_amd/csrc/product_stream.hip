// Products with few rows a group, as units of product_stream.h, and the launch of every product.
#include <algorithm>

#include "product_choice.h"
#include "product_stream.h"

namespace craft {
namespace {

// Four waves: eight of half the ring each, with blocks of 32 rows, take the same time within 3 % for one to 16 tokens and a gated decode
// step, 78 us in place of 72 for 250 rows on 32 experts in bf16, and 52 in place of 58 for 400 gated ones on 30 in 8 bits.
constexpr int kStreamWaves = 4, kThreads = 64 * kStreamWaves;

// Blocks of ROWS rows before each group, in LDS: [G + 1].  Every wave works them out for itself and stores the same, so
// that no barrier is needed: a wave reads what it has written.
template <int ROWS> static __device__ __forceinline__ void count_blocks(const ProductArgs &a, int32_t *before) {
    const int lane = threadIdx.x & 63;
    int32_t sum = 0;
    for (int32_t g0 = 0; g0 < a.G; g0 += 64) {
        const int32_t g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < a.G) group_rows(a, g, lo, hi);
        int32_t n[1] = {(int32_t)((hi - lo + ROWS - 1) / ROWS)};
        wave_sums(n);
        if (g < a.G) before[g + 1] = sum + n[0];
        sum += __builtin_amdgcn_readlane(n[0], 63);
    }
    before[0] = 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// MOST: 16-row fragments of a block, 1 or 4; SPLIT: 1 or all of a workgroup's waves
template <int FMT, bool GATED, int CF, int MOST, int SPLIT>
__global__ __launch_bounds__(kThreads) void product_stream_kernel(ProductArgs a) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int RING = kStreamLds / kStreamWaves, ROWS = 16 * MOST;
    __shared__ __attribute__((aligned(16))) unsigned char smem[kStreamLds];
    __shared__ int32_t before[kMostGroups + 1];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t cols = (a.N + 16 * CF - 1) / (16 * CF);
    count_blocks<ROWS>(a, before);
    const int64_t units = (int64_t)before[a.G] * cols;
    // neighbouring units (the blocks of rows of the same columns, then the next columns) on one XCD
    const int64_t place = (int64_t)(blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8;
    const int64_t first = SPLIT > 1 ? place : place * kStreamWaves + wave, step = (int64_t)gridDim.x * (SPLIT > 1 ? 1 : kStreamWaves);
    for (int64_t w = first; w < units; w += step) {
        int32_t lo = 0, hi = a.G;                  // before[lo] * cols <= w < before[hi] * cols
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if ((int64_t)before[mid] * cols <= w) lo = mid; else hi = mid;
        }
        const int32_t blocks = before[hi] - before[lo];
        const int64_t in = w - (int64_t)before[lo] * cols;
        int64_t r0, r1;
        group_rows(a, lo, r0, r1);
        Unit u;
        u.group = __builtin_amdgcn_readfirstlane(lo);
        u.n0 = __builtin_amdgcn_readfirstlane((int32_t)(in / blocks) * 16 * CF);
        u.row0 = r0 + (in % blocks) * ROWS;
        u.rows = __builtin_amdgcn_readfirstlane((int32_t)min((int64_t)ROWS, r1 - u.row0));
        unsigned char *const ring = smem + wave * RING;
        acc_t *const part = reinterpret_cast<acc_t *>(smem);
        if constexpr (MOST == 1) {
            stream_unit<FMT, GATED, CF, 1, SPLIT, RING>(a, u, ring, part);
        } else {
            if (u.rows <= 16) stream_unit<FMT, GATED, CF, 1, SPLIT, RING>(a, u, ring, part);
            else if (u.rows <= 32) stream_unit<FMT, GATED, CF, 2, SPLIT, RING>(a, u, ring, part);
            else stream_unit<FMT, GATED, CF, 4, SPLIT, RING>(a, u, ring, part);
        }
    }
}

template <int FMT, bool GATED, int CF, int MOST> void launch_split(const ProductArgs &a, hipStream_t s) {
    // most blocks of rows that there can be
    const int64_t blocks = a.M / (16 * MOST) + std::min<int64_t>(a.M, a.G);
    const int64_t units = blocks * ((a.N + 16 * CF - 1) / (16 * CF));
    const bool alone = units >= (int64_t)a.num_cu * kStreamWaves;
    const int64_t need = alone ? (units + kStreamWaves - 1) / kStreamWaves : units;
    const dim3 grid((unsigned)((std::min<int64_t>(need, a.num_cu) + 7) / 8 * 8));
    if (alone) hipLaunchKernelGGL((product_stream_kernel<FMT, GATED, CF, MOST, 1>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((product_stream_kernel<FMT, GATED, CF, MOST, kStreamWaves>), grid, dim3(kThreads), 0, s, a);
}
template <int FMT, bool GATED> hipError_t launch_stream(const ProductArgs &a, hipStream_t s) {
    constexpr int WIDE = GATED ? 1 : 2;
    if (a.M <= 16) launch_split<FMT, GATED, WIDE, 1>(a, s);
    else launch_split<FMT, GATED, WIDE, 4>(a, s);
    return hipGetLastError();
}

template <bool GATED> hipError_t launch_format(const ProductArgs &a, hipStream_t s) {
    if (a.format == CRAFT_I8) return launch_stream<CRAFT_I8, GATED>(a, s);
    if (a.format == CRAFT_BF16) return launch_stream<CRAFT_BF16, GATED>(a, s);
    return launch_stream<CRAFT_F32, GATED>(a, s);
}

}  // namespace

hipError_t launch_product(const ProductArgs &a, hipStream_t s) {
    if (a.M <= 0) return hipSuccess;
    const ProductChoice c = product_choice(a);
    if (c.height) {
        if (a.format == CRAFT_I8) return launch_product_tiles_i8(a, c.width, c.height, s);
        if (a.format == CRAFT_BF16) return launch_product_tiles_bf16(a, c.width, c.height, s);
        return launch_product_tiles_f32(a, c.width, c.height, s);
    }
    return a.up ? launch_format<true>(a, s) : launch_format<false>(a, s);
}

}  // namespace craft
