// Products with few rows a group: the weights are read once, straight from memory into operand registers, and the
// contraction is shared among the waves of a workgroup.
//
// A unit is 16 CF columns of one group's matrix (gated: of both) against up to 64 of its rows.  Wave v of the
// workgroup takes slabs v, v + WAVES, .. of 128 bytes along the contraction, a ring of them on their way; the waves'
// sums meet in LDS and are added in wave order (integers: any order gives the same).
#include <algorithm>

#include "product_stream.h"

namespace craft {
namespace {

// Units' row blocks before each group, in LDS: [G + 1].
template <int THREADS> static __device__ __forceinline__ void count_blocks(const ProductArgs &a, int32_t *before, int32_t *scratch) {
    // a thread's run of neighbouring groups, then a scan over threads
    const int32_t each = (a.G + THREADS - 1) / THREADS, first = min((int32_t)threadIdx.x * each, a.G), last = min(first + each, a.G);
    int32_t sum = 0;
    for (int32_t g = first; g < last; ++g) {
        int64_t lo, hi;
        group_rows(a, g, lo, hi);
        const int32_t n = (int32_t)((hi - lo + kUnitRows - 1) / kUnitRows);
        before[g] = n;
        sum += n;
    }
    scratch[threadIdx.x] = sum;
    __syncthreads();
    for (int d = 1; d < THREADS; d *= 2) {
        const int32_t add = (int)threadIdx.x >= d ? scratch[threadIdx.x - d] : 0;
        __syncthreads();
        scratch[threadIdx.x] += add;
        __syncthreads();
    }
    int32_t at = scratch[threadIdx.x] - sum;
    for (int32_t g = first; g < last; ++g) {
        const int32_t n = before[g];
        before[g] = at;
        at += n;
    }
    if (threadIdx.x == THREADS - 1) before[a.G] = scratch[THREADS - 1];
    __syncthreads();
}

template <int FMT, bool GATED, int CF, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void product_stream_kernel(ProductArgs a) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    __shared__ acc_t part[WAVES * CF * (GATED ? 2 : 1) * 4 * 64];
    __shared__ int32_t before[kMostGroups + 1], scratch[64 * WAVES];
    const int32_t cols = (a.N + 16 * CF - 1) / (16 * CF);
    count_blocks<64 * WAVES>(a, before, scratch);
    const int64_t units = (int64_t)before[a.G] * cols;
    for (int64_t w = blockIdx.x; w < units; w += gridDim.x) {
        const int32_t block = (int32_t)(w / cols);
        int32_t lo = 0, hi = a.G;                  // before[lo] <= block < before[hi]
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (before[mid] <= block) lo = mid; else hi = mid;
        }
        int64_t first, last;
        group_rows(a, lo, first, last);
        Unit u;
        u.group = __builtin_amdgcn_readfirstlane(lo);
        u.n0 = __builtin_amdgcn_readfirstlane((int32_t)(w % cols) * 16 * CF);
        u.row0 = first + (int64_t)(block - before[lo]) * kUnitRows;
        u.rows = __builtin_amdgcn_readfirstlane((int32_t)min((int64_t)kUnitRows, last - u.row0));
        if (u.rows <= 16) stream_unit<FMT, GATED, CF, 1, WAVES>(a, u, part);
        else if (u.rows <= 32) stream_unit<FMT, GATED, CF, 2, WAVES>(a, u, part);
        else stream_unit<FMT, GATED, CF, 4, WAVES>(a, u, part);
    }
}

template <int FMT, bool GATED>
hipError_t launch_stream(const ProductArgs &a, hipStream_t s) {
    const int64_t blocks = a.M / kUnitRows + std::min<int64_t>(a.M, a.G);
    const int64_t grid = std::min<int64_t>(blocks * ((a.N + 15) / 16), (int64_t)a.num_cu * 4);
    hipLaunchKernelGGL((product_stream_kernel<FMT, GATED, 1, 4>), dim3((unsigned)grid), dim3(256), 0, s, a);
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
    const bool near = a.src ? a.x_rows * a.x_stride < (int64_t)1 << 32 : a.x_stride < (int64_t)1 << 24;
    if (near && a.row_bytes >= 128 && a.M >= 128 && a.M / a.G >= 16) {
        const int64_t nt = (a.N + (a.up ? 127 : 255)) / (a.up ? 128 : 256);
        int32_t height = 256;
        while (height > 64 && a.M / height * nt < a.num_cu) height -= 64;
        if (a.format == CRAFT_I8) return launch_product_tiles_i8(a, height, s);
        if (a.format == CRAFT_BF16) return launch_product_tiles_bf16(a, height, s);
        return launch_product_tiles_f32(a, height, s);
    }
    return a.up ? launch_format<true>(a, s) : launch_format<false>(a, s);
}

}  // namespace craft
