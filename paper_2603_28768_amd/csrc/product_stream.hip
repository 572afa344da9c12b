// Products with few rows a group, as units of product_stream.h, and which kernel takes a product.
#include <algorithm>
#include <cmath>

#include "product_stream.h"

namespace craft {
namespace {

constexpr int kThreads = 64 * kStreamWaves;

// Row blocks of 64 before each group, in LDS: [G + 1].  Every wave works them out for itself and stores the same, so
// that no barrier is needed: a wave reads what it has written.
static __device__ __forceinline__ void count_blocks(const ProductArgs &a, int32_t *before) {
    const int lane = threadIdx.x & 63;
    int32_t sum = 0;
    for (int32_t g0 = 0; g0 < a.G; g0 += 64) {
        const int32_t g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < a.G) group_rows(a, g, lo, hi);
        int32_t n = (int32_t)((hi - lo + kUnitRows - 1) / kUnitRows);
        n = sum + wave_sums(n);
        if (g < a.G) before[g + 1] = n;
        sum = __builtin_amdgcn_readlane(n, 63);
    }
    before[0] = 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// ROWS: most 16-row fragments of a unit
template <int FMT, bool GATED, int CF, int ROWS, int SPLIT>
__global__ __launch_bounds__(kThreads) void product_stream_kernel(ProductArgs a) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    __shared__ __attribute__((aligned(16))) unsigned char smem[kStreamWaves * kRingBytes];
    __shared__ int32_t before[kMostGroups + 1];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t cols = (a.N + 16 * CF - 1) / (16 * CF);
    count_blocks(a, before);
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
        u.row0 = r0 + (in % blocks) * kUnitRows;
        u.rows = __builtin_amdgcn_readfirstlane((int32_t)min((int64_t)kUnitRows, r1 - u.row0));
        unsigned char *const ring = smem + wave * kRingBytes;
        acc_t *const part = reinterpret_cast<acc_t *>(smem);
        if (ROWS == 1 || u.rows <= 16) stream_unit<FMT, GATED, CF, 1, SPLIT>(a, u, ring, part);
        else if (u.rows <= 32) stream_unit<FMT, GATED, CF, 2, SPLIT>(a, u, ring, part);
        else stream_unit<FMT, GATED, CF, 4, SPLIT>(a, u, ring, part);
    }
}

template <int FMT, bool GATED, int CF, int ROWS> void launch_split(const ProductArgs &a, int64_t blocks, hipStream_t s) {
    const int64_t units = blocks * ((a.N + 16 * CF - 1) / (16 * CF));
    const bool alone = units >= (int64_t)a.num_cu * kStreamWaves;
    const int64_t need = alone ? (units + kStreamWaves - 1) / kStreamWaves : units;
    const dim3 grid((unsigned)((std::min<int64_t>(need, a.num_cu) + 7) / 8 * 8));
    if (alone) hipLaunchKernelGGL((product_stream_kernel<FMT, GATED, CF, ROWS, 1>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((product_stream_kernel<FMT, GATED, CF, ROWS, kStreamWaves>), grid, dim3(kThreads), 0, s, a);
}
template <int FMT, bool GATED> hipError_t launch_stream(const ProductArgs &a, hipStream_t s) {
    // most row blocks that there can be
    const int64_t blocks = a.M / kUnitRows + std::min<int64_t>(a.M, a.G);
    constexpr int WIDE = GATED ? 1 : 2;
    if (a.M <= 16) launch_split<FMT, GATED, WIDE, 1>(a, blocks, s);
    else launch_split<FMT, GATED, WIDE, 4>(a, blocks, s);
    return hipGetLastError();
}

template <bool GATED> hipError_t launch_format(const ProductArgs &a, hipStream_t s) {
    if (a.format == CRAFT_I8) return launch_stream<CRAFT_I8, GATED>(a, s);
    if (a.format == CRAFT_BF16) return launch_stream<CRAFT_BF16, GATED>(a, s);
    return launch_stream<CRAFT_F32, GATED>(a, s);
}

}  // namespace

// Size of the tiles: the one whose rounds take the least.  A slab of a tile of FW x FX fragments a wave takes 88 FW + 26 FW FX
// cycles (measured: 0.39 us at 4 x 4, 0.87 at 8 x 4, 1.2 at 8 x 8), a tile 12000 and 150 for every product of fragments
// beside its slabs.  How rows are spread over groups only the GPU knows: a third of a tile more for each is assumed.  Behind the first
// round tiles end at different times.
void product_tile_size(const ProductArgs &a, int32_t *width, int32_t *height) {
    const int64_t slabs = (a.row_bytes + 127) / 128, per_element = a.format == CRAFT_F32 ? 4 : 1;
    double best = 0;
    for (int fw = 8; fw >= 4; fw -= 4)
        for (int fx = fw; fx >= 2; --fx) {
            if (fx == 3) continue;
            const int64_t columns = 32 * fw / (a.up ? 2 : 1), nt = (a.N + columns - 1) / columns;
            const double rows = a.G == 1 ? (double)((a.M + 32 * fx - 1) / (32 * fx)) : (double)a.M / (32 * fx) + 0.35 * a.G;
            const double rounds = rows * nt / a.num_cu;
            const double made = rounds <= 1 ? 1 : a.G == 1 ? std::ceil(rounds) : rounds + 0.6;
            const double slab = 88.0 * fw + 26.0 * fw * fx * per_element;
            const double time = made * (slabs * slab + 12000 + 150 * fw * fx);
            if (best == 0 || time < best) {
                best = time;
                *width = 32 * fw;
                *height = 32 * fx;
            }
        }
}

hipError_t launch_product(const ProductArgs &a, hipStream_t s) {
    if (a.M <= 0) return hipSuccess;
    const bool near = a.src ? a.x_rows * a.x_stride < (int64_t)1 << 32 : a.x_stride < (int64_t)1 << 24;
    if (near && a.row_bytes >= 128 && a.M >= 128 && a.M / a.G >= 16) {
        int32_t width = 256, height = 256;
        product_tile_size(a, &width, &height);
        if (a.format == CRAFT_I8) return launch_product_tiles_i8(a, width, height, s);
        if (a.format == CRAFT_BF16) return launch_product_tiles_bf16(a, width, height, s);
        return launch_product_tiles_f32(a, width, height, s);
    }
    return a.up ? launch_format<true>(a, s) : launch_format<false>(a, s);
}

}  // namespace craft
