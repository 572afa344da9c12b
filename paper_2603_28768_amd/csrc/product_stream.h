// Few rows of a group against its weights, which are read once, straight from memory into operand registers.
//
// A unit is 16 CF columns of one group's matrix (gated: of both) against up to 64 of its rows.  Wave v of the
// workgroup takes slabs v, v + WAVES, .. of 128 bytes along the contraction, a ring of them on their way; the waves'
// sums meet in LDS and are added in wave order (integers: any order gives the same).
#pragma once

#include "product.h"

namespace craft {

constexpr int kUnitRows = 64;

struct Unit {
    int32_t group, n0, rows;       // rows of this unit, 1 .. 64
    int64_t row0;                  // its first row among the M
};

template <int FMT, bool GATED, int CF, int RF, int WAVES>
static __device__ __forceinline__ void stream_unit(const ProductArgs &a, const Unit &u, typename Numbers<FMT>::acc_t *part) {
    typedef Numbers<FMT> T;
    typedef typename T::acc_t acc_t;
    constexpr int MATS = GATED ? 2 : 1, WF = CF * MATS;
    constexpr int D = WF + RF <= 2 ? 6 : WF + RF <= 4 ? 3 : 2;        // slabs of a wave on their way
    const int lane = threadIdx.x & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t KB = a.row_bytes, slabs = (KB + 127) >> 7;
    bytes_t w[WF], x[RF];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
        const bytes_t mat = (bytes_t)(a.off ? (m ? +a.up : +a.w)[u.group] : a.w_one);
#pragma unroll
        for (int c = 0; c < CF; ++c) w[m * CF + c] = mat + (int64_t)min(u.n0 + 16 * c + r16, a.N - 1) * KB;
    }
#pragma unroll
    for (int g = 0; g < RF; ++g) {
        const int64_t t = token_of(a, u.row0 + min(16 * g + r16, u.rows - 1));
        x[g] = (bytes_t)a.x + (t < 0 ? 0 : t) * a.x_stride;
    }
    raw_t wv[D][2][WF], xv[D][2][RF];
    // (pieces past the rows: read from inside them, replaced by zeros below)
    auto load = [&](int d, int32_t slab) __attribute__((always_inline)) {
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const int32_t at = min(slab * 128 + step * 64 + q * 16, KB - 16);
#pragma unroll
            for (int c = 0; c < WF; ++c) wv[d][step][c] = *(pieces_t)(w[c] + at);
#pragma unroll
            for (int g = 0; g < RF; ++g) xv[d][step][g] = *(pieces_t)(x[g] + at);
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
                const scales_t ws = (scales_t)(a.off ? (m ? +a.up_scale : +a.w_scale)[u.group] : a.w_one_scale);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[m][e] = (float)s[m][e] * xs * ws[min(col + e, a.N - 1)];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[m][e] = s[m][e];
            }
        }
        if constexpr (GATED)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = (FMT == CRAFT_F32 || a.out_dtype == CRAFT_F32 ? silu_f32(v[0][e]) : silu_bf16(v[0][e])) * v[1][e];
        if (t < 0)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = 0.0f;
        store_columns(a, p, col, v[0], a.out_whole);
    }
}

}  // namespace craft
