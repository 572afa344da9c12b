// Rows to 8-bit integers with a scale each: scale = max |x| / 127, code = the integer nearest to the fp32 quotient x / scale.
//
// A row is read once and stays in registers between its maximum and its codes: LANES lanes share it in units of 16
// elements (32 or 64 bytes in, one 16-byte store out), lane l taking units l, l + LANES, ..  Bound by HBM.
#include <algorithm>

#include "product.h"

namespace craft {
namespace {

constexpr float kSmallestScale = 0x1p-126f;    // the smallest normal number: no scale is a denormal one

// The fp32 quotient of 16 elements by the row's scale, rounded to integers.  y is the correctly rounded reciprocal: a
// product by it, corrected by its remainder twice, is the correctly rounded quotient (Markstein), in five instructions
// where a division takes ten.  The remainders of very small rows would be lost below the smallest number: TINY divides.
// Adding 1.5 x 2^23 rounds to an integer, ties to even, and leaves it in the lowest bits.
template <bool TINY> static __device__ __forceinline__ uint32_t code_bits(float x, float s, float y) {
    float q = x * y;
    q = fmaf(fmaf(-s, q, x), y, q);
    q = fmaf(fmaf(-s, q, x), y, q);
    if (TINY) q = x / s;
    return __builtin_bit_cast(uint32_t, q + 12582912.0f);
}
static __device__ __forceinline__ uint32_t bytes_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

template <bool F32> struct UnitOf {
    static constexpr int RAW = F32 ? 4 : 2;        // 16-byte pieces of a unit
    raw_t v[RAW];
    __device__ __forceinline__ void load(const unsigned char *p) {
#pragma unroll
        for (int i = 0; i < RAW; ++i) v[i] = *reinterpret_cast<const raw_t *>(p + 16 * i);
    }
    // the largest magnitude's bits: as integers NaN > infinity > any number
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < RAW; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (F32) m = max(m, v[i][j] & 0x7fffffffu);
                else m = max(m, max(v[i][j] & 0x7fff0000u, (v[i][j] << 16) & 0x7fffffffu));
            }
        return m;
    }
    __device__ __forceinline__ float element(int e) const {
        // (a word of its own first: a bit cast of a vector's element takes the vector's first)
        const uint32_t w = F32 ? v[e >> 2][e & 3] : v[e >> 3][(e >> 1) & 3];
        const uint32_t bits = F32 ? w : e & 1 ? w & 0xffff0000u : w << 16;
        return __builtin_bit_cast(float, bits);
    }
    template <bool TINY> __device__ __forceinline__ void store(int8_t *out, float s, float y) const {
        raw_t c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c[i] = bytes_of(code_bits<TINY>(element(4 * i), s, y), code_bits<TINY>(element(4 * i + 1), s, y),
                            code_bits<TINY>(element(4 * i + 2), s, y), code_bits<TINY>(element(4 * i + 3), s, y));
        *reinterpret_cast<raw_t *>(out) = c;
    }
};

struct RowScale {
    float stored, s, y;                            // s, y: what the codes are made with
    bool finite, tiny;
};
static __device__ __forceinline__ RowScale scale_of(uint32_t bits) {
    RowScale r;
    r.finite = bits < 0x7f800000u;
    const float most = __builtin_bit_cast(float, bits);
    r.s = !r.finite || bits == 0 ? 1.0f : fmaxf(most / 127.0f, kSmallestScale);
    r.stored = r.finite ? r.s : __builtin_bit_cast(float, 0x7fc00000u);
    r.y = 1.0f / r.s;
    r.tiny = r.s < 0x1p-90f;
    return r;
}

// CHUNKS units a lane, one row for every LANES lanes: 16 or 64 of a wave, or the whole workgroup.
template <bool F32, int LANES, int CHUNKS>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeI8Args a) {
    constexpr int64_t PER = 256 / LANES;
    const int64_t row = (int64_t)blockIdx.x * PER + threadIdx.x / LANES;
    const int lane = (int)threadIdx.x % LANES, units = a.K >> 4;
    if (row >= a.rows) return;
    const unsigned char *x = a.x + row * a.x_stride;
    UnitOf<F32> u[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) u[c].load(x + (int64_t)min(lane + c * LANES, units - 1) * (F32 ? 64 : 32));
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) m = max(m, u[c].largest());
#pragma unroll
    for (int d = 1; d < LANES && d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d, LANES < 64 ? LANES : 64));
    if constexpr (LANES > 64) {
        __shared__ uint32_t most[4];
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(most[0], most[1]), max(most[2], most[3]));
    }
    const RowScale r = scale_of(m);
    if (lane == 0) a.scale[row] = r.stored;
    int8_t *out = a.codes + row * a.K;
    // (one branch for all of a row: divided for everywhere and chosen from, 20011 bf16 rows of 7168 take 97 us
    // in place of 78)
    if (__builtin_expect(r.finite && !r.tiny, 1)) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = lane + c * LANES;
            if (at < units) u[c].template store<false>(out + (int64_t)at * 16, r.s, r.y);
        }
    } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int at = lane + c * LANES;
            if (at >= units) continue;
            if (r.finite) u[c].template store<true>(out + (int64_t)at * 16, r.s, r.y);
            else *reinterpret_cast<raw_t *>(out + (int64_t)at * 16) = raw_t{};
        }
    }
}

// Rows of any length: a workgroup each, read twice.
template <bool F32> __global__ __launch_bounds__(256) void quantize_long_kernel(QuantizeI8Args a, int64_t first) {
    __shared__ uint32_t most[4];
    const int64_t row = first + blockIdx.x;
    const int units = a.K >> 4;
    const unsigned char *x = a.x + row * a.x_stride;
    UnitOf<F32> u;
    uint32_t m = 0;
    for (int at = threadIdx.x; at < units; at += 256) {
        u.load(x + (int64_t)at * (F32 ? 64 : 32));
        m = max(m, u.largest());
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
    __syncthreads();
    const RowScale r = scale_of(max(max(most[0], most[1]), max(most[2], most[3])));
    if (threadIdx.x == 0) a.scale[row] = r.stored;
    int8_t *out = a.codes + row * a.K;
    for (int at = threadIdx.x; at < units; at += 256) {
        u.load(x + (int64_t)at * (F32 ? 64 : 32));
        if (r.finite && !r.tiny) u.template store<false>(out + (int64_t)at * 16, r.s, r.y);
        else if (r.finite) u.template store<true>(out + (int64_t)at * 16, r.s, r.y);
        else *reinterpret_cast<raw_t *>(out + (int64_t)at * 16) = raw_t{};
    }
}

constexpr int64_t kMostGroupsLaunched = (1ll << 32) / 256 - 1;     // a launch has fewer than 2^32 threads

template <bool F32, int LANES, int CHUNKS> void launch_rows(QuantizeI8Args a, hipStream_t s) {
    constexpr int64_t PER = 256 / LANES;
    for (int64_t left = a.rows; left > 0; left -= kMostGroupsLaunched * PER) {
        a.rows = std::min(left, kMostGroupsLaunched * PER);
        hipLaunchKernelGGL((quantize_rows_kernel<F32, LANES, CHUNKS>), dim3((unsigned)((a.rows + PER - 1) / PER)), dim3(256), 0, s, a);
        a.x += a.rows * a.x_stride;
        a.codes += a.rows * a.K;
        a.scale += a.rows;
    }
}
template <bool F32> void launch_type(const QuantizeI8Args &a, hipStream_t s) {
    const int units = a.K >> 4;
    // Short rows share a wave where there are enough to fill the GPU: fewer lanes are idle at a row's end.
    const bool many = a.rows >= 8192;
    if (units <= 16) launch_rows<F32, 16, 1>(a, s);
    else if (many && units <= 32) launch_rows<F32, 16, 2>(a, s);
    else if (many && units <= 48) launch_rows<F32, 16, 3>(a, s);
    else if (units <= 64) launch_rows<F32, 64, 1>(a, s);
    else if (many && units <= 96) launch_rows<F32, 16, 6>(a, s);
    else if (units <= 128) launch_rows<F32, 64, 2>(a, s);
    else if (units <= 192) launch_rows<F32, 64, 3>(a, s);
    else if (units <= 256) launch_rows<F32, 64, 4>(a, s);
    else if (units <= 320) launch_rows<F32, 64, 5>(a, s);
    else if (units <= 384) launch_rows<F32, 64, 6>(a, s);
    else if (units <= 448) launch_rows<F32, 64, 7>(a, s);
    else if (units <= 512) launch_rows<F32, 64, 8>(a, s);
    else if (units <= 768) launch_rows<F32, 256, 3>(a, s);
    else if (units <= 1024) launch_rows<F32, 256, 4>(a, s);
    else if (units <= 2048) launch_rows<F32, 256, 8>(a, s);
    else
        for (int64_t r = 0; r < a.rows; r += kMostGroupsLaunched)
            hipLaunchKernelGGL((quantize_long_kernel<F32>), dim3((unsigned)std::min(kMostGroupsLaunched, a.rows - r)), dim3(256), 0, s, a, r);
}

}  // namespace

hipError_t launch_quantize_i8(const QuantizeI8Args &a, hipStream_t s) {
    if (a.rows <= 0) return hipSuccess;
    if (a.dtype == CRAFT_F32) launch_type<true>(a, s);
    else launch_type<false>(a, s);
    return hipGetLastError();
}

}  // namespace craft
