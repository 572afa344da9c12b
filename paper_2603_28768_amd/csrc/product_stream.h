// Few rows of a group against its weights, which are read once.
//
// A unit is 16 CF columns of one group's matrix (gated: of both) against up to 16 RF of its rows.  One wave has it by itself,
// or SPLIT waves of a workgroup share it along the contraction: wave v takes slabs v, v + SPLIT, .. of 128 bytes a row, and
// the waves' sums meet in LDS and are added in wave order (integers: any order gives the same).
// Weights and rows travel straight into LDS, whole lines of eight rows a request, into a ring of slabs that is the wave's own:
// no barrier, a wave waits for its own requests by count.  Where lanes load fragments of row-major matrices themselves (16
// lines for every 16 lanes) a CU gets 38 GB/s of its L1, which weights and rows have to share; this way 123.
#pragma once

#include "product.h"

namespace craft {

constexpr int kStreamLds = 144 << 10;              // of a workgroup, shared among its waves

struct Unit {
    int32_t group, n0, rows;       // rows of this unit, 1 .. 16 RF
    int64_t row0;                  // its first row among the M
};

// ring: this wave's part of LDS;  part: room for the sums of SPLIT waves, LDS that nobody reads any more once all are here
template <int FMT, bool GATED, int CF, int RF, int SPLIT, int RING>
static __device__ __forceinline__ void stream_unit(const ProductArgs &a, const Unit &u, unsigned char *ring, typename Numbers<FMT>::acc_t *part) {
    typedef Numbers<FMT> T;
    typedef typename T::acc_t acc_t;
    constexpr int MATS = GATED ? 2 : 1, WF = CF * MATS, NR = WF + RF, SLAB = NR * 2048, REQ = 2 * NR;
    constexpr int D0 = RING / SLAB, D = D0 < 8 ? D0 : 8;
    static_assert(D >= 2 && D * REQ <= 63, "slabs on their way");
    const int lane = threadIdx.x & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), mine = SPLIT > 1 ? wave : 0;
    const int32_t KB = a.row_bytes, slabs = (KB + 127) >> 7;
    // chunk j of an operand is eight rows; pieces of a row in the order piece ^ (row & 7)
    const uint32_t piece = (uint32_t)min((((lane & 7) ^ ((lane >> 3) & 7)) * 16), KB - 16);
    uint32_t woff[2 * CF];
    ubase_t wbase[MATS], x[2 * RF];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
        wbase[m] = uniform_base((a.off ? (m ? +a.up : +a.w)[u.group] : a.w_one) + (int64_t)u.n0 * KB);
#pragma unroll
    for (int j = 0; j < 2 * CF; ++j) woff[j] = (uint32_t)min(8 * j + (lane >> 3), a.N - 1 - u.n0) * (uint32_t)KB + piece;
#pragma unroll
    for (int j = 0; j < 2 * RF; ++j) {
        const int64_t p = u.row0 + min(8 * j + (lane >> 3), u.rows - 1), t = a.src ? token_of(a, p) : p;
        x[j] = a.x + (t < 0 ? 0 : t) * a.x_stride + piece;
    }
    const uint32_t lds0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)ring);
    const uint32_t fo = (uint32_t)(r16 * 128 + ((q ^ (lane & 7)) & 7) * 16);
    typedef const raw_t __attribute__((address_space(3))) *frag_t;
    // the last slab ends with the rows; what the one before it has is cut away (rows of less than a slab: what is behind them)
    auto request = [&](int32_t slab, uint32_t at) __attribute__((always_inline)) {
        const uint32_t k = (uint32_t)__builtin_amdgcn_readfirstlane(max(min(slab * 128, KB - 128), 0));
#pragma unroll
        for (int j = 0; j < 2 * WF; ++j) {
            dma_to(at + (uint32_t)(j * 1024));
            asm volatile("s_nop 0");
            dma_request(wbase[j / (2 * CF)] + k, woff[j % (2 * CF)]);
        }
#pragma unroll
        for (int j = 0; j < 2 * RF; ++j) {
            dma_to(at + (uint32_t)((2 * WF + j) * 1024));
            asm volatile("s_nop 0");
            dma_request_at(x[j] + k);
        }
    };
    acc_t acc[WF][RF];
#pragma unroll
    for (int c = 0; c < WF; ++c)
#pragma unroll
        for (int g = 0; g < RF; ++g) acc[c][g] = acc_t{};
    const int32_t n = (slabs - mine + SPLIT - 1) / SPLIT;
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < n) request(mine + d * SPLIT, lds0 + (uint32_t)(d * SLAB));
    uint32_t slot = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (i + D <= n) dma_wait<(D - 1) * REQ>();
        else dma_wait<0>();
        const int32_t slab = mine + i * SPLIT;
        raw_t wv[2][WF], xv[2][RF];
#pragma unroll
        for (int step = 0; step < 2; ++step) {
            const uint32_t from = lds0 + slot + (fo ^ (step ? 64u : 0u));
#pragma unroll
            for (int g = 0; g < RF; ++g) xv[step][g] = *(frag_t)(uintptr_t)(from + (uint32_t)((WF + g) * 2048));
#pragma unroll
            for (int c = 0; c < WF; ++c) wv[step][c] = *(frag_t)(uintptr_t)(from + (uint32_t)(c * 2048));
        }
        if (slab + 1 == slabs && (KB & 127)) {
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const int at = step * 64 + q * 16;
                const bool gone = KB >= 128 ? at < slabs * 128 - KB : at >= KB;
#pragma unroll
                for (int c = 0; c < WF; ++c) wv[step][c] = gone ? raw_t{} : wv[step][c];
#pragma unroll
                for (int g = 0; g < RF; ++g) xv[step][g] = gone ? raw_t{} : xv[step][g];
            }
        }
#pragma unroll
        for (int step = 0; step < 2; ++step)
#pragma unroll
            for (int c = 0; c < WF; ++c)
#pragma unroll
                for (int g = 0; g < RF; ++g) T::multiply(wv[step][c], xv[step][g], acc[c][g]);
        // what was in the slot is in registers
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + D < n) request(slab + D * SPLIT, lds0 + slot);
        slot = slot + SLAB < D * SLAB ? slot + SLAB : 0;
    }
    if (SPLIT > 1) {
        __syncthreads();                           // every wave has read its last slab
#pragma unroll
        for (int c = 0; c < WF; ++c)
#pragma unroll
            for (int g = 0; g < RF; ++g) part[((wave * WF + c) * RF + g) * 64 + lane] = acc[c][g];
        __syncthreads();
    }
    // element v of lane l is column 4 (l >> 4) + v and row l & 15 of its fragment
    const bool accurate = FMT == CRAFT_F32 || a.out_dtype == CRAFT_F32;
#pragma unroll
    for (int c = 0; c < CF; ++c)
#pragma unroll
        for (int g = 0; g < RF; ++g) {
            if (SPLIT > 1 && (c * RF + g) % SPLIT != wave) continue;
            acc_t s[MATS];
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
                if (SPLIT > 1) {
                    s[m] = part[((m * CF + c) * RF + g) * 64 + lane];
#pragma unroll
                    for (int v = 1; v < SPLIT; ++v) s[m] += part[((v * WF + m * CF + c) * RF + g) * 64 + lane];
                } else {
                    s[m] = acc[m * CF + c][g];
                }
            }
            const int32_t row = 16 * g + r16, col = u.n0 + 16 * c + 4 * q;
            if (row >= u.rows || col >= a.N) continue;
            const int64_t p = u.row0 + row, t = a.src ? token_of(a, p) : p;
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
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (GATED) v[0][e] = (accurate ? silu_f32(v[0][e]) : silu_bf16(v[0][e])) * v[1][e];
                v[0][e] = t < 0 ? 0.0f : v[0][e];
            }
            store_columns(a, p, col, v[0], a.out_whole);
        }
    if (SPLIT > 1) __syncthreads();                // the sums have been read: LDS may be filled again
}

}  // namespace craft
