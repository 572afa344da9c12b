// Products with few rows a group, as units of product_stream.h, and which kernel takes a product.
#include <algorithm>
#include <cmath>

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

// Which kernel, and the size of its tiles: what is expected to take the least time, from sizes that the host knows.  How rows are
// spread over groups only the GPU knows.  Fitted to times of 70 drawn products of 6 to 3700 rows (1 to 68 groups, every type), of
// which the choice takes 1.008 of the better kernel's time in the geometric mean; units up to 127 rows or 15 a group and tiles
// beyond took 1.13.
struct Sizes {
    double rows, groups, columns, slabs;           // groups: those that can have rows
    double matrix;                                 // cycles of a slab's matrix instructions, relative to 16 bits
    double weights;                                // ns that the weights take out of HBM
};
Sizes sizes_of(const ProductArgs &a) {
    Sizes z;
    z.rows = (double)a.M;
    z.groups = (double)std::min<int64_t>(a.M, a.G);
    z.columns = a.N;
    z.slabs = (a.row_bytes + 127) / 128;
    z.matrix = a.format == CRAFT_F32 ? 4 : 1;
    z.weights = z.groups * a.N * a.row_bytes * (a.up ? 2 : 1) / 5000;
    return z;
}
// ns of units: their bytes at 60 GB/s a CU, or their matrix instructions; 2 us for a unit that four waves share, 4 to 5.5 for
// four of a wave each, whose results go out at the same time.
double stream_time(const ProductArgs &a, const Sizes &z) {
    const double blocks = a.G == 1 ? std::ceil(z.rows / 64) : std::max(z.groups, z.rows / 64 + 0.5 * z.groups);
    const double rows = z.rows / blocks, fx = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const double units = blocks * std::ceil(z.columns / (a.up ? 16 : 32));
    const double bytes = z.slabs * (2 + fx) * 2048, matrix = z.slabs * 4 * fx * 16 / 2 * (z.matrix > 1 ? 8 : 1);
    double time;
    if (units >= 4.0 * a.num_cu) time = std::ceil(units / (4.0 * a.num_cu)) * (std::max(4 * bytes / 60, matrix) + 3500 + 500 * fx);
    else time = std::ceil(units / a.num_cu) * (std::max(bytes / 60, matrix / 4) + 2000);
    return std::max(time, z.weights);
}
// ns of tiles.  A slab of a tile of FW x FX fragments a wave takes 88 FW + 26 FW FX cycles (0.39 us at 4 x 4, 0.87 at 8 x 4, 1.2 at
// 8 x 8), a tile 12000 and 150 for every product of fragments beside its slabs, at 2 GHz.  A third of a tile more for each group is
// assumed, and that behind the first round tiles end at different times; groups of 64 rows in the mean: low tiles.
double tile_time(const ProductArgs &a, const Sizes &z, int32_t *width, int32_t *height) {
    double best = 0;
    for (int fw = 8; fw >= 4; fw -= 4)
        for (int fx = fw; fx >= 2; --fx) {
            if (fx == 3) continue;
            const double columns = std::ceil(z.columns / (32 * fw / (a.up ? 2 : 1)));
            const double rows = a.G == 1 ? std::ceil(z.rows / (32 * fx)) : z.rows / (32 * fx) + 0.35 * a.G;
            const double rounds = rows * columns / a.num_cu;
            const double made = rounds <= 1 ? 1 : a.G == 1 ? std::ceil(rounds) : rounds + 0.6;
            const double time = made * (z.slabs * (88 * fw + 26 * fw * fx * z.matrix) + 12000 + 150 * fw * fx) / 2;
            if (best == 0 || time < best) {
                best = time;
                *width = 32 * fw;
                *height = 32 * fx;
            }
        }
    if (z.rows / a.G <= 64) {
        const double rounds = z.groups * std::ceil(z.columns / (a.up ? 64 : 128)) / a.num_cu, fx = z.rows / a.G <= 32 ? 1 : 2;
        best = (rounds < 2 ? std::ceil(rounds) : rounds + 0.5) * (z.slabs * (352 + 104 * fx * z.matrix) + 12500) / 2;
    }
    return std::max(best, z.weights * 5000 / 4500);
}

}  // namespace

hipError_t launch_product(const ProductArgs &a, hipStream_t s) {
    if (a.M <= 0) return hipSuccess;
    const bool near = a.src ? a.x_rows * a.x_stride < (int64_t)1 << 32 : a.x_stride < (int64_t)1 << 24;
    if (near && a.row_bytes >= 128 && a.M > 16) {
        const Sizes z = sizes_of(a);
        int32_t width = 0, height = 0;
        if (tile_time(a, z, &width, &height) < stream_time(a, z)) {
            if (a.format == CRAFT_I8) return launch_product_tiles_i8(a, width, height, s);
            if (a.format == CRAFT_BF16) return launch_product_tiles_bf16(a, width, height, s);
            return launch_product_tiles_f32(a, width, height, s);
        }
    }
    return a.up ? launch_format<true>(a, s) : launch_format<false>(a, s);
}

}  // namespace craft
