// Products with few rows a group: the weights are read once, straight from memory into operand registers, and the
// contraction is shared among the waves of a workgroup.
//
// A unit is 16 CF columns of one group's matrix (gated: of both) against up to 64 of its rows.  Wave v of the
// workgroup takes slabs v, v + WAVES, .. of 128 bytes along the contraction, a ring of them on their way; the waves'
// sums meet in LDS and are added in wave order (integers: any order gives the same).
#include <algorithm>

#include "product.h"

namespace craft {
namespace {

constexpr int kUnitRows = 64;

struct Unit {
    int32_t group, n0, rows;       // rows of this unit, 1 .. 64
    int64_t row0;                  // its first row among the M
};

// Units' row blocks before each group, in LDS: [G + 1].
template <int THREADS> static __device__ void count_blocks(const ProductArgs &a, int32_t *before, int32_t *scratch) {
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

// fp32 results: the library exponential; those rounded to bf16: the hardware one (2^-21 off where silu matters)
static __device__ __forceinline__ float silu_of(float g, bool exact) { return g / (1.0f + (exact ? expf(-g) : __expf(-g))); }

template <int FMT, bool GATED, int CF, int RF, int WAVES>
static __device__ __forceinline__ void stream_unit(const ProductArgs &a, const Unit &u, typename Numbers<FMT>::acc_t *part) {
    typedef Numbers<FMT> T;
    typedef typename T::acc_t acc_t;
    constexpr int MATS = GATED ? 2 : 1, WF = CF * MATS;
    constexpr int D = WF + RF <= 2 ? 6 : WF + RF <= 4 ? 3 : 2;        // slabs of a wave on their way
    const int lane = threadIdx.x & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t KB = a.row_bytes, slabs = (KB + 127) >> 7;
    const unsigned char *w[WF], *x[RF];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
        const unsigned char *mat = a.off ? (m ? a.up : a.w)[u.group] : a.w_one;
#pragma unroll
        for (int c = 0; c < CF; ++c) w[m * CF + c] = mat + (int64_t)min(u.n0 + 16 * c + r16, a.N - 1) * KB;
    }
#pragma unroll
    for (int g = 0; g < RF; ++g) {
        const int64_t t = token_of(a, u.row0 + min(16 * g + r16, u.rows - 1));
        x[g] = a.x + (t < 0 ? 0 : t) * a.x_stride;
    }
    raw_t wv[D][2][WF], xv[D][2][RF];
    // (pieces past the rows: read from inside them, replaced by zeros below)
    auto load = [&](int d, int32_t slab) __attribute__((always_inline)) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const int32_t at = min(slab * 128 + step * 64 + q * 16, KB - 16);
#pragma unroll
            for (int c = 0; c < WF; ++c) wv[d][step][c] = *reinterpret_cast<const raw_t *>(w[c] + at);
#pragma unroll
            for (int g = 0; g < RF; ++g) xv[d][step][g] = *reinterpret_cast<const raw_t *>(x[g] + at);
        }
    };
    acc_t acc[WF][RF];
#pragma unroll
    for (int c = 0; c < WF; ++c)
#pragma unroll
        for (int g = 0; g < RF; ++g) acc[c][g] = acc_t{};
#pragma unroll
    for (int d = 0; d < D; ++d) load(d, min(wave + d * WAVES, slabs));
    for (int32_t s0 = wave; s0 < slabs; s0 += D * WAVES) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const int32_t slab = s0 + d * WAVES;
            if (slab >= slabs) break;
            if (slab * 128 + 128 > KB) {
#pragma unroll
                for (int step = 0; step < 2; ++step) {
                    const bool past = slab * 128 + step * 64 + q * 16 >= KB;
#pragma unroll
                    for (int c = 0; c < WF; ++c) wv[d][step][c] = past ? raw_t{} : wv[d][step][c];
#pragma unroll
                    for (int g = 0; g < RF; ++g) xv[d][step][g] = past ? raw_t{} : xv[d][step][g];
                }
            }
#pragma unroll
            for (int step = 0; step < 2; ++step)
#pragma unroll
                for (int c = 0; c < WF; ++c)
#pragma unroll
                    for (int g = 0; g < RF; ++g) T::multiply(wv[d][step][c], xv[d][step][g], acc[c][g]);
            load(d, min(slab + D * WAVES, slabs));
        }
    }
    __syncthreads();                               // the last unit's sums have been read
#pragma unroll
    for (int c = 0; c < WF; ++c)
#pragma unroll
        for (int g = 0; g < RF; ++g) part[((wave * WF + c) * RF + g) * 64 + lane] = acc[c][g];
    __syncthreads();
    // element v of lane l is column 4 (l >> 4) + v and row l & 15 of its fragment
    for (int f = wave; f < CF * RF; f += WAVES) {
        const int c = f / RF, g = f % RF;
        acc_t s[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            s[m] = part[((m * CF + c) * RF + g) * 64 + lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) s[m] += part[((v * WF + m * CF + c) * RF + g) * 64 + lane];
        }
        const int32_t row = 16 * g + r16, col = u.n0 + 16 * c + 4 * q;
        if (row >= u.rows || col >= a.N) continue;
        const int64_t p = u.row0 + row, t = token_of(a, p);
        float v[MATS][4];
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            if constexpr (FMT == CRAFT_I8) {
                const float xs = a.x_scale[t < 0 ? 0 : t];
                const float *ws = a.off ? (m ? a.up_scale : a.w_scale)[u.group] : a.w_one_scale;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[m][e] = (float)s[m][e] * xs * ws[min(col + e, a.N - 1)];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[m][e] = s[m][e];
            }
        }
        if constexpr (GATED)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = silu_of(v[0][e], FMT == CRAFT_F32 || a.out_dtype == CRAFT_F32) * v[1][e];
        if (t < 0)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = 0.0f;
        store_columns(a, p, col, v[0], a.out_whole);
    }
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
    return a.up ? launch_format<true>(a, s) : launch_format<false>(a, s);
}

}  // namespace craft
