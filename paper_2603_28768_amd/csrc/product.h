// Matrix products whose operands are both stored row by row along the contraction, out = x w^T, of three kinds of numbers:
// fp32, bf16 (fp32 sums) and 8-bit integers (32-bit integer sums, exact), alone or grouped by expert.
//
// All kernels see rows as bytes: an operand fragment is 16 rows x 64 bytes, lane l holding bytes 16 (l >> 4) .. + 15 of row
// l & 15.  That is 16 codes, 8 bf16 values or 4 floats of the contraction; which of them meet in one matrix
// instruction does not matter as long as both operands agree.
#pragma once

#include "ffn_common.h"
#include "kernels.h"

namespace craft {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float pf32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 pbf16x8_t __attribute__((ext_vector_type(8)));
typedef unsigned int raw_t __attribute__((ext_vector_type(4)));        // 16 bytes of a row

// Addresses read from a table in memory: said to be global, they are else read as flat ones, which wait for LDS as well.
typedef const float __attribute__((address_space(1))) *scales_t;

template <int FMT> struct Numbers;
template <> struct Numbers<CRAFT_F32> {
    typedef pf32x4_t acc_t;
    static __device__ __forceinline__ void multiply(raw_t w, raw_t x, acc_t &c) {
        const pf32x4_t a = __builtin_bit_cast(pf32x4_t, w), b = __builtin_bit_cast(pf32x4_t, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    }
};
template <> struct Numbers<CRAFT_BF16> {
    typedef pf32x4_t acc_t;
    static __device__ __forceinline__ void multiply(raw_t w, raw_t x, acc_t &c) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pbf16x8_t, w), __builtin_bit_cast(pbf16x8_t, x), c, 0, 0, 0);
    }
};
template <> struct Numbers<CRAFT_I8> {
    typedef i32x4_t acc_t;
    static __device__ __forceinline__ void multiply(raw_t w, raw_t x, acc_t &c) {
        c = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, w), __builtin_bit_cast(i32x4_t, x), c, 0, 0, 0);
    }
};

// silu for fp32 results, and for those rounded to bf16 right after: the hardware's exponential and reciprocal (2^-21 off
// where silu matters), with numerator and denominator scaled down alike, since a reciprocal below 2^-126 becomes zero
// (g < -87.3, where silu times a large second factor still is a number).
static __device__ __forceinline__ float silu_f32(float g) { return g / (1.0f + expf(-g)); }
static __device__ __forceinline__ float silu_bf16(float g) { return g * 0x1p-8f * __builtin_amdgcn_rcpf(fmaf(__expf(-g), 0x1p-8f, 0x1p-8f)); }

// Four neighbouring columns of one row into the result, whatever its alignment: `whole` where rows and columns allow
// one store.
static __device__ __forceinline__ void store_columns(const ProductArgs &a, int64_t row, int32_t col, const float (&v)[4], bool whole) {
    if (a.out_dtype == CRAFT_BF16) {
        uint16_t *p = static_cast<uint16_t *>(a.out) + row * a.out_stride + col;
        const uint2 two = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
        if (whole && col + 4 <= a.N) {
            *reinterpret_cast<uint2 *>(p) = two;
        } else {
            const uint32_t u[2] = {two.x, two.y};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < a.N) p[i] = (uint16_t)(u[i >> 1] >> (16 * (i & 1)));
        }
    } else {
        float *p = static_cast<float *>(a.out) + row * a.out_stride + col;
        if (whole && col + 4 <= a.N) {
            *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < a.N) p[i] = v[i];
        }
    }
}

// Row p of the products is this row of x; -1: the permutation names none, and the result is zeros.  Only where there is one.
static __device__ __forceinline__ int32_t token_of(const ProductArgs &a, int64_t p) {
    const int32_t s = a.src[p];
    // s / k: the product with 2^(31 + l) / k rounded up, l = ceil(log2 k), is exact for 31 bits
    const int32_t t = a.k == 1 ? s : (int32_t)(__umulhi((uint32_t)s, a.k_magic) >> a.k_shift);
    return s >= 0 && t < a.x_rows ? t : -1;
}

// Rows of group g, inside [0, M) whatever the offsets are.
static __device__ __forceinline__ void group_rows(const ProductArgs &a, int32_t g, int64_t &lo, int64_t &hi) {
    if (!a.off) {
        lo = 0;
        hi = a.M;
        return;
    }
    const int64_t l = a.off[g], h = a.off[g + 1];
    lo = l < 0 ? 0 : l < a.M ? l : a.M;
    hi = h < lo ? lo : h < a.M ? h : a.M;
}

// Inclusive sums over the lanes of a wave.
template <int DPP, int ROWS> static __device__ __forceinline__ int32_t lane_before(int32_t x) {
    return __builtin_amdgcn_update_dpp(0, x, DPP, ROWS, 0xf, false);
}
// Several at a time: an instruction across lanes reads what was written two instructions earlier at the soonest.
template <int N> static __device__ __forceinline__ void wave_sums(int32_t (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x111, 0xf>(x[i]);     // one, two, four, eight lanes up a row of 16
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x112, 0xf>(x[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x114, 0xf>(x[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x118, 0xf>(x[i]);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x142, 0xa>(x[i]);     // a row's last lane into the next row, the second one's
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] += lane_before<0x143, 0xc>(x[i]);     // into the upper half
}

}  // namespace craft
