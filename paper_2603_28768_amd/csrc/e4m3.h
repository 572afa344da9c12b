// Quantisation to OCP FP8 E4M3 with a scale per row, as device functions: of expert weights (quant.hip) and of
// cached keys and values (kv_cache.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace craft {

// Nearest E4M3 magnitude to a >= 0, ties to the even mantissa, saturating at 448.  The value
// grid inside one binade is 2^(e-3), so the mantissa is a rounded quotient; below 2^-6 the
// grid is 2^-9 throughout.  rintf rounds halves to even, which is the rule for the code too
// (the last mantissa bit is the last bit of the code, and a carry into the next binade lands
// on its first, even, value).
static __device__ __forceinline__ uint32_t e4m3_magnitude(float a) {
    if (!(a < 448.0f)) return 0x7e;
    if (a < 0.015625f) return (uint32_t)rintf(a * 512.0f);          // 0..8; 8 is the smallest normal
    const int e = (int)((__float_as_uint(a) >> 23) & 0xff) - 127;   // floor(log2 a), a is normal here
    const int n = (int)rintf(ldexpf(a, 3 - e));                     // 8..16
    const uint32_t code = n == 16 ? (uint32_t)(e + 8) << 3 : ((uint32_t)(e + 7) << 3) | (uint32_t)(n - 8);
    return code > 0x7e ? 0x7e : code;
}

// A row's scale and what dividing by it takes.  The code of an element is decided by the
// correctly rounded fp32 quotient w / s.  With y the correctly rounded reciprocal of s and
// q = w y, the sum q + (w - s q) y is that quotient (Markstein 1990) unless an intermediate
// leaves the normal range: with s between 2^-60 and 2^60 none does for a quotient of 2^-10 or
// more, and everything below is code 0 either way.  Three operations instead of the ten or so
// of a division, which is what keeps the kernels below bound by memory.  Other rows (an
// infinity in them, or next to nothing) take the division.
struct RowScale {
    float s, inv;
    bool fast;
};
static __device__ __forceinline__ RowScale row_scale(float amax) {
    RowScale r;
    r.s = amax > 0.0f ? amax / 448.0f : 1.0f;
    r.inv = 1.0f / r.s;
    r.fast = r.s >= 0x1p-60f && r.s <= 0x1p60f;
    return r;
}
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
static __device__ __forceinline__ float low_value(uint32_t w) { return __uint_as_float(w << 16); }
static __device__ __forceinline__ float high_value(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
static __device__ __forceinline__ float max_abs(float m, const u32x4_t &w) {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = fmaxf(fmaxf(m, fabsf(low_value(w[i]))), fabsf(high_value(w[i])));
    return m;
}
// The codes of 4 bf16 values (two words, low half first).
static __device__ __forceinline__ uint32_t four_codes(uint32_t w0, uint32_t w1, const RowScale &r) {
    const float a[4] = {fabsf(low_value(w0)), fabsf(high_value(w0)), fabsf(low_value(w1)), fabsf(high_value(w1))};
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float q0 = a[i] * r.inv;
        q[i] = fminf(fmaf(fmaf(-r.s, q0, a[i]), r.inv, q0), 448.0f);      // a NaN saturates too
    }
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);        // nearest, ties to even
    c = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
    // the sign bits: the high bytes of the four halves
    return (uint32_t)c | (__builtin_amdgcn_perm(w1, w0, 0x07050301u) & 0x80808080u);
}
static __device__ __forceinline__ uint32_t four_codes_divided(uint32_t w0, uint32_t w1, float s) {
    const float v[4] = {low_value(w0), high_value(w0), low_value(w1), high_value(w1)};
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float q = v[i] / s;
        c |= (e4m3_magnitude(fabsf(q)) | (__float_as_uint(q) >> 31 << 7)) << (8 * i);
    }
    return c;
}
static __device__ __forceinline__ u32x2_t eight_codes(const u32x4_t &w, const RowScale &r) {
    u32x2_t c;
    if (r.fast) {
        c[0] = four_codes(w[0], w[1], r);
        c[1] = four_codes(w[2], w[3], r);
    } else {
        c[0] = four_codes_divided(w[0], w[1], r.s);
        c[1] = four_codes_divided(w[2], w[3], r.s);
    }
    return c;
}

}  // namespace craft
