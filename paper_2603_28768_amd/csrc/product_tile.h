// Products with many rows a group: tiles of up to 256 rows of x against 256 rows of the weights, one workgroup of four
// waves (2 x 2 over the tile) per CU.
//
// Both operands go from memory straight into LDS (loads that write LDS, ffn_common.h) in slabs of 128 bytes a row, whole
// lines: a CU gets 123 GB/s that way, and 38 where lanes load operand fragments of row-major weights themselves (16 rows a
// request; the same tile 265 us so, 8192 x 4096 x 7168).  An LDS row is unpadded, its eight 16-byte pieces in the order piece ^
// (row & 7), so that the reads of a fragment hit every bank once.  A slab is two steps of 64 bytes.  While one step is multiplied,
// all fragments of the next are read into the other set of registers: behind the first step of a slab its stages are free
// again.  x of the slab that takes its place is requested in the second step, its weights in the first step of the next slab.
// Every memory instruction is dealt out behind a matrix instruction of its own.
//
// A group's rows are shared evenly among as few tiles of at most `height` rows as hold them, in whole fragments of 32.  Groups of up
// to 64 rows, which stream their weights through one CU at what that gets out of HBM, have tiles of 128 weight rows with up to six stages.
// The list has the tallest tiles first.  Groups that overlap can have more tiles than were launched for; those are cut otherwise.
#pragma once

#include <algorithm>
#include <type_traits>

#include "product.h"

namespace craft {
namespace {

constexpr int kThreads = 256;
constexpr int kSlab = 128;                         // bytes of the contraction
constexpr int kTileLds = 160 << 10;                // all there is
// Stages of the weights and of x.  Weights come from HBM the first time, x mostly from L2: where what is left holds a stage of
// weights besides, they have one more.
template <int FW, int FX> constexpr int both_stages() { return kTileLds / ((FW + FX) * 32 * kSlab); }
template <int FW, int FX> constexpr bool more_weights() { return both_stages<FW, FX>() == 2 && (3 * FW + 2 * FX) * 32 * kSlab <= kTileLds; }
template <int FW, int FX> constexpr int x_stages() { return both_stages<FW, FX>() < 6 ? both_stages<FW, FX>() : 6; }
template <int FW, int FX> constexpr int w_stages() { return more_weights<FW, FX>() ? 3 : x_stages<FW, FX>(); }
constexpr int kLowColumns = 4;                     // fragments of weights a wave for groups of few rows

template <int FMT> static __device__ __forceinline__ void multiply_in_place(raw_t w, raw_t x, typename Numbers<FMT>::acc_t &c) {
    if constexpr (FMT == CRAFT_I8) {
        asm("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
    } else if constexpr (FMT == CRAFT_BF16) {
        asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(w), "v"(x));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t p = w[e], q = x[e];
            asm("v_mfma_f32_16x16x4_f32 %0, %1, %2, %0" : "+a"(c) : "v"(p), "v"(q));
        }
    }
}

struct Tile {
    int32_t group, rows, n0;       // n0: first column of the result
    int64_t row0;
};

// FW, FX: 16-row fragments of weights and of x per wave; the tile is 32 FW columns (gated: 16 FW) x 32 FX rows.
template <int FMT, bool GATED, int FW, int FX>
static __device__ __forceinline__ void product_tile(const ProductArgs &a, const Tile &t, unsigned char *smem, int tid) {
    typedef typename Numbers<FMT>::acc_t acc_t;
    constexpr int M = FW * FX, NR = FW + FX, SW = w_stages<FW, FX>(), SX = x_stages<FW, FX>();
    constexpr uint32_t WSTAGE = FW * 32 * kSlab, XSTAGE = FX * 32 * kSlab, XRING = SW * WSTAGE;
    static_assert(((SW == SX && SX >= 3) || (SX == 2 && SW == 3)) && XRING + SX * XSTAGE <= kTileLds && SX * NR <= 63, "stages");
    const int lane = tid & 63, q = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t KB = a.row_bytes, nk = (KB + kSlab - 1) / kSlab;
    // Chunk 4 i + wave, eight rows of an operand, is this wave's i-th.  In front of LDS: weights, then x.
    const uint32_t piece = (uint32_t)(((lane & 7) ^ ((lane >> 3) & 7)) * 16);
    const bool gather = a.src != nullptr;
    const ubase_t xbase = uniform_base(gather ? a.x : a.x + t.row0 * a.x_stride);
    uint32_t woff[FW], xoff[FX];
#pragma unroll
    for (int i = 0; i < FX; ++i) {
        const int r = min(8 * (4 * i + wave) + (lane >> 3), t.rows - 1);
        const int32_t tok = gather ? token_of(a, t.row0 + r) : r;
        xoff[i] = (uint32_t)max(tok, 0) * (uint32_t)a.x_stride + piece;
    }
    // what a thread's row of the tile is multiplied by; goes to LDS when there is time for it
    const int64_t my_row = gather ? token_of(a, t.row0 + min(tid, t.rows - 1)) : t.row0 + min(tid, t.rows - 1);
    const float my_scale = FMT == CRAFT_I8 ? a.x_scale[my_row < 0 ? 0 : my_row] : 1.0f;
    // Gated: 16 rows of gate are followed by the 16 of up of the same columns; the first two waves fetch gate's.
    const unsigned char *mat;
    if constexpr (GATED) {
        const unsigned char *const *side = a.w;
        if (wave >= 2) side = a.up;
        mat = side[t.group];
    } else {
        mat = a.off ? a.w[t.group] : a.w_one;
    }
    const ubase_t wbase = uniform_base(mat + (int64_t)t.n0 * KB);
    auto column = [](int r) { return GATED ? (r >> 5) * 16 + (r & 15) : r; };
#pragma unroll
    for (int i = 0; i < FW; ++i) woff[i] = (uint32_t)min(column(8 * (4 * i + wave) + (lane >> 3)), a.N - 1 - t.n0) * (uint32_t)KB + piece;

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const uint32_t lds_wave = lds0 + (uint32_t)__builtin_amdgcn_readfirstlane(wave * 1024);
    const uint32_t fo = lds0 + (uint32_t)(r16 * 128 + ((q ^ (lane & 7)) & 7) * 16);
    const uint32_t fw0 = fo + (uint32_t)((wave >> 1) * FW * 2048), fx0 = fo + XRING + (uint32_t)((wave & 1) * FX * 2048);
    typedef const raw_t __attribute__((address_space(3))) *frag_t;

    raw_t wv[2][FW], xv[2][FX];
    acc_t acc[FW][FX];
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int g = 0; g < FX; ++g) acc[f][g] = acc_t{};

    // where slab ks begins in a row: the last one ends with it, and what the one before has is cut away
    auto at = [&](int ks) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readfirstlane(min(ks * kSlab, KB - kSlab)); };
    // request i of a slab's x, or of its weights, into a stage of theirs
    auto aim = [&](auto X, int i, uint32_t stage) __attribute__((always_inline)) {
        dma_to(lds_wave + (X.value ? XRING : 0u) + stage + (uint32_t)(4096 * i));
    };
    auto request = [&](auto X, int i, uint32_t k) __attribute__((always_inline)) {
        if constexpr (X.value) dma_request(xbase + k, xoff[i < FX ? i : 0]);
        else dma_request(wbase + k, woff[i < FW ? i : 0]);
    };
    // x's fragments first, the next products start with those
    struct From { uint32_t x, w; };                // one register each, fragments at constant offsets from them
    auto from = [&](int step, uint32_t w, uint32_t x) __attribute__((always_inline)) {
        From p = {(fx0 ^ (step ? 64u : 0u)) + x, (fw0 ^ (step ? 64u : 0u)) + w};
        asm volatile("" : "+v"(p.x), "+v"(p.w));
        return p;
    };
    auto fetch = [&](int set, int j, const From &p) __attribute__((always_inline)) {
        if (j < FX) xv[set][j < FX ? j : 0] = *(frag_t)(uintptr_t)(p.x + (uint32_t)(j * 2048));
        else wv[set][j < FX ? 0 : j - FX] = *(frag_t)(uintptr_t)(p.w + (uint32_t)((j - FX) * 2048));
    };
    // bytes of the last slab that the one before it has already; a matrix instruction may read what a vector instruction wrote
    // two cycles later
    auto cut = [&](int set) __attribute__((always_inline)) {
        const bool gone = set * 64 + q * 16 < nk * kSlab - KB;
#pragma unroll
        for (int g = 0; g < FX; ++g) {
            xv[set][g] = gone ? raw_t{} : xv[set][g];
            asm volatile("s_nop 1" : "+v"(xv[set][g]));
        }
#pragma unroll
        for (int f = 0; f < FW; ++f) {
            wv[set][f] = gone ? raw_t{} : wv[set][f];
            asm volatile("s_nop 1" : "+v"(wv[set][f]));
        }
    };
    // One step: set STEP multiplied, the other one read from stages w and x; and, if REQ, this slab's requests at k into
    // stage `to`: weights in the first step, x in the second, so that they are as far apart as they can be (all of them in one step:
    // 8192 x 4096 x 14336 in zeros 304 us).
    auto step_of = [&](auto STEP, auto REQ, uint32_t w, uint32_t x, uint32_t to, uint32_t k) __attribute__((always_inline)) {
        constexpr int set = STEP.value, R = !REQ.value ? 0 : set ? FX : FW, OPS = NR + 2 * R;
        const std::integral_constant<bool, set == 1> of_x;
        const From p = from(set ^ 1, w, x);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            multiply_in_place<FMT>(wv[set][m / FX], xv[set][m % FX], acc[m / FX][m % FX]);
            // spread over seven eighths of the step: what is read has to be there when the next one begins
#pragma unroll
            for (int o = min(m * OPS * 8 / (7 * M), OPS); o < min((m + 1) * OPS * 8 / (7 * M), OPS); ++o) {
                // a request's address, a fragment, the request: a load may not follow its M0 at once
                const int i = o / 3;
                if (i < R) {
                    if (o % 3 == 0) aim(of_x, i, to);
                    else if (o % 3 == 1) fetch(set ^ 1, i, p);
                    else request(of_x, i, k);
                } else {
                    fetch(set ^ 1, o - 2 * R, p);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const std::integral_constant<int, 0> step0;
    const std::integral_constant<int, 1> step1;
    const std::true_type with;
    const std::false_type without;
    const bool cuts = nk * kSlab != KB;

    auto start = [&](auto X, int j) __attribute__((always_inline)) {
        if (j < nk) {
            const uint32_t k = at(j);
#pragma unroll
            for (int i = 0; i < (X.value ? FX : FW); ++i) {
                aim(X, i, j * (X.value ? XSTAGE : WSTAGE));
                asm volatile("s_nop 0");
                request(X, i, k);
            }
        }
    };
#pragma unroll
    for (int j = 0; j < SX; ++j) {
        start(with, j);
        if (j < SW - 1) start(without, j);
    }
    if (nk >= SX) dma_wait<(SX - 1) * FX + (SW - 2) * FW>();
    else dma_wait<0>();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NR; ++j) fetch(0, j, from(0, 0, 0));
    uint32_t hw = 0, hx = 0;                       // stages of slab ks
    int ks = 0;
    auto next_w = [&](uint32_t v) { return v + WSTAGE < SW * WSTAGE ? v + WSTAGE : 0; };
    auto next_x = [&](uint32_t v) { return v + XSTAGE < SX * XSTAGE ? v + XSTAGE : 0; };
    auto last_w = [&](uint32_t v) { return v > 0 ? v - WSTAGE : (SW - 1) * WSTAGE; };
    // In slab ks, weights of slab ks + SW - 1 are requested into the stage of slab ks - 1, behind the barrier x of slab ks + SX into
    // that of slab ks.  At the barrier, behind the first step, all of slab ks is in registers of every wave and slab ks + 1 has landed:
    // what was requested behind its x and its weights may be on its way.
    constexpr int BEHIND_X = (SX - 1) * FW + (SX - 2) * FX, BEHIND_W = (SW - 2) * NR;
    constexpr int BEHIND = BEHIND_X < BEHIND_W ? BEHIND_X : BEHIND_W;
    for (; ks + SX < nk; ++ks) {
        const uint32_t tw = next_w(hw), tx = next_x(hx);
        step_of(step0, with, hw, hx, last_w(hw), at(ks + SW - 1));
        dma_wait<BEHIND>();
        __syncthreads();
        step_of(step1, with, tw, tx, hx, at(ks + SX));
        hw = tw;
        hx = tx;
    }
    if (SW == SX && ks + SX == nk) {               // the last weights are still to be requested
        const uint32_t tw = next_w(hw), tx = next_x(hx);
        step_of(step0, with, hw, hx, last_w(hw), at(ks + SW - 1));
        dma_wait<BEHIND>();
        __syncthreads();
        step_of(step1, without, tw, tx, 0, 0);
        hw = tw;
        hx = tx;
        ++ks;
    }
    for (; ks < nk; ++ks) {
        const uint32_t tw = next_w(hw), tx = next_x(hx);
        const bool last = ks + 1 == nk;
        if (last && cuts) cut(0);
        step_of(step0, without, hw, hx, 0, 0);
        if (ks + 2 < nk) dma_wait<FW>();           // the last weights were requested behind what is needed now
        else dma_wait<0>();
        __syncthreads();
        if (last && cuts) cut(1);
        step_of(step1, without, tw, tx, 0, 0);     // (behind the last slab: read and not used)
        hw = tw;
        hx = tx;
    }
    // a matrix instruction's result is read: idle cycles, then every accumulator through a statement behind them
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int f = 0; f < FW; ++f)
#pragma unroll
        for (int g = 0; g < FX; ++g) asm volatile("" : "+a"(acc[f][g]));

    // element v of lane l is column 4 (l >> 4) + v and row l & 15 of its fragment
    constexpr int SIDES = GATED ? 2 : 1;
    const int32_t col0 = t.n0 + column((wave >> 1) * FW * 16) + 4 * q;
    float ws[FW][4];
    if (FMT == CRAFT_I8) {
        const scales_t s0 = (scales_t)(a.off ? a.w_scale[t.group] : a.w_one_scale), s1 = GATED ? (scales_t)a.up_scale[t.group] : s0;
#pragma unroll
        for (int f = 0; f < FW; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int32_t c = min(col0 + f / SIDES * 16 + e, a.N - 1);
                if (f & (SIDES - 1)) ws[f][e] = s1[c];
                else ws[f][e] = s0[c];
            }
    }
    float *const row_scale = reinterpret_cast<float *>(smem + kTileLds - 4096);
    uint8_t *const row_live = smem + kTileLds - 2048;
    // By way of LDS, 16 rows at a time and each wave for itself, so that a store covers whole lines (16 rows of 32 bytes a
    // request: 8 us a tile).  While 16 rows come back from there the next are worked out.  Stores are of 16 bytes whatever the
    // alignment; a lane at the matrix' edge stores its columns one by one.
    auto results = [&](auto BF16) __attribute__((always_inline)) {
        constexpr bool bf16 = BF16.value;
        typedef typename std::conditional<bf16, uint16_t, float>::type out_t;
        typedef out_t piece_t __attribute__((ext_vector_type(16 / sizeof(out_t)), aligned(sizeof(out_t))));
        constexpr int ES = (int)sizeof(out_t), COLS = 16 * FW / SIDES, ROWB = COLS * ES, PITCH = ROWB + 16, BUFFER = 16 * PITCH;
        constexpr int PER = ROWB / 16, EACH = 16 / ES, PASSES = 16 * PER / 64, ROWS = 64 / PER;     // pieces of a row; elements of a piece; rows of a pass
        static_assert(4 * 2 * BUFFER <= kTileLds - 4096 && PER <= 64, "rows of results");
        unsigned char *const mine = smem + wave * (2 * BUFFER);
        const int32_t first = t.n0 + (wave >> 1) * COLS, row0 = (wave & 1) * FX * 16;
        int l0 = lane;
        asm volatile("" : "+v"(l0));
        const int r = l0 / PER, c = l0 % PER * EACH;
        const bool full = t.rows == 32 * FX && t.n0 + 2 * COLS <= a.N;      // the whole tile is there
        out_t *p = static_cast<out_t *>(a.out) + first + c + (t.row0 + row0 + r) * a.out_stride;
        const int64_t pass = ROWS * a.out_stride;
        raw_t v[PASSES];
        auto put = [&](int g) __attribute__((always_inline)) {
            int l = lane;                          // (places are worked out here, not in front of everything for all of it)
            asm volatile("" : "+v"(l));
            unsigned char *const to = mine + (g & 1) * BUFFER + (l & 15) * PITCH + (l >> 4) * 4 * ES;
            const int row = row0 + 16 * g + (l & 15);
            const float xs = FMT == CRAFT_I8 ? row_scale[row] : 1.0f;
#pragma unroll
            for (int f = 0; f < FW; f += SIDES) {
                float y[SIDES][4];
#pragma unroll
                for (int m = 0; m < SIDES; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[m][e] = FMT == CRAFT_I8 ? (float)acc[f + m][g][e] * xs * ws[f + m][e] : (float)acc[f + m][g][e];
                if constexpr (GATED)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[0][e] = (bf16 ? silu_bf16(y[0][e]) : silu_f32(y[0][e])) * y[SIDES - 1][e];
                if constexpr (bf16) *reinterpret_cast<uint2 *>(to + f / SIDES * 32) = make_uint2(bf16_pair(y[0][0], y[0][1]), bf16_pair(y[0][2], y[0][3]));
                else *reinterpret_cast<float4 *>(to + f / SIDES * 64) = make_float4(y[0][0], y[0][1], y[0][2], y[0][3]);
            }
            if (gather && !row_live[row])          // (seldom)
#pragma unroll 1
                for (int f = 0; f < FW / SIDES; ++f)
                    for (int e = 0; e < 4; ++e) reinterpret_cast<out_t *>(to + f * 16 * ES)[e] = 0;
            __builtin_amdgcn_sched_barrier(0);
        };
        put(0);
#pragma unroll
        for (int g = 0; g < FX; ++g) {
            // (the wave's own rows: its reads follow its writes)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const unsigned char *from = mine + (g & 1) * BUFFER + r * PITCH + c * ES;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) v[i] = *reinterpret_cast<const raw_t *>(from + i * ROWS * PITCH);
            __builtin_amdgcn_sched_barrier(0);
            if (g + 1 < FX) put(g + 1);
            if (full) {
#pragma unroll
                for (int i = 0; i < PASSES; ++i) *reinterpret_cast<piece_t *>(p + i * pass) = __builtin_bit_cast(piece_t, v[i]);
            } else {
#pragma unroll
                for (int i = 0; i < PASSES; ++i)
                    if (row0 + 16 * g + i * ROWS + r < t.rows) {
                        out_t *to = p + i * pass;
                        if (first + c + EACH <= a.N) *reinterpret_cast<piece_t *>(to) = __builtin_bit_cast(piece_t, v[i]);
                        else
#pragma unroll 1
                            for (int e = 0; first + c + e < a.N; ++e) to[e] = reinterpret_cast<const out_t *>(from + i * ROWS * PITCH)[e];
                    }
            }
            p += PASSES * pass;
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    __syncthreads();                               // every wave has read the last slab
    row_live[tid] = my_row >= 0;
    if (FMT == CRAFT_I8) row_scale[tid] = my_scale;
    __syncthreads();
    if (FMT != CRAFT_F32 && a.out_dtype == CRAFT_BF16) results(with);
    else results(without);
}

// How a group's rows are cut: kFew into one low tile, else into tiles of `height` rows (the last one what is left), the classes by height.
constexpr int kClasses = 4, kFew = 3, kFewRows = 64;
struct Cut {
    int32_t kind, height, count;
};
static __device__ __forceinline__ Cut cut_rows(int32_t rows, int32_t most) {
    if (rows <= kFewRows) return {kFew, kFewRows, rows > 0};
    const uint32_t r = (uint32_t)rows, m = (uint32_t)most, tiles = (r + m - 1) / m, height = ((r + tiles - 1) / tiles + 31) / 32 * 32;
    return {height > 192 ? 0 : height > 128 ? 1 : 2, (int32_t)height, (int32_t)((r + height - 1) / height)};
}
// 64 groups, one a lane: their rows and how they are cut.
struct Groups {
    int64_t lo, hi;
    Cut cut;
};
static __device__ __forceinline__ Groups groups_at(const ProductArgs &a, int32_t g, int32_t height) {
    Groups r = {0, 0, {}};
    if (g < a.G) group_rows(a, g, r.lo, r.hi);
    r.cut = cut_rows((int32_t)(r.hi - r.lo), height);
    return r;
}
static __device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}

// Item i of a group's m x nt tiles: blocks of 8 x 8, column by column inside a block, so that the tiles that run at one
// time need few rows of either operand between them.
static __device__ __forceinline__ void place(uint32_t i, uint32_t m, uint32_t nt, int32_t &row, int32_t &col) {
    const uint32_t band = i / (8 * nt), r0 = band * 8, rj = min(8u, m - r0), in = i - r0 * nt;
    const uint32_t block = in / (rj * 8), rest = in - block * rj * 8, across = rest / rj;
    row = (int32_t)(r0 + rest - across * rj);
    col = (int32_t)(block * 8 + across);
}

// Every step-th tile from `first` on, of a list without classes: 64 rows, 32 kLowColumns columns.  A loop costs little with the
// registers that such tiles need, and what they take is not what counts here.  The arguments, the kernel's first, are read
// anew for every tile: kept, they would take scalar registers from the other tiles' path too.
template <int FMT, bool GATED>
static __device__ __forceinline__ void overlapping_tiles(unsigned char *smem, int tid, int64_t first, int64_t step) {
    constexpr int LOW = 32 * kLowColumns / (GATED ? 2 : 1);
    for (int64_t w = first;; w += step) {
        auto args = __builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(args));
        const ProductArgs a = *(const ProductArgs *)args;
        const int32_t nlow = (a.N + LOW - 1) / LOW, lane = tid & 63;
        const int64_t place_in = w / nlow;
        Tile t = {};
        int64_t behind_last = 0;
        int32_t run_up = 0;
        bool found = false;
        for (int32_t g0 = 0; g0 < a.G && !found; g0 += 64) {
            const int32_t g = g0 + lane;
            int64_t lo = 0, hi = 0;
            if (g < a.G) group_rows(a, g, lo, hi);
            const int32_t count = (int32_t)((hi - lo + kFewRows - 1) / kFewRows);
            int32_t upto[1] = {count};
            wave_sums(upto);
            upto[0] += run_up;
            const uint64_t behind = __ballot(upto[0] > place_in);
            if (behind) {
                const int at = __builtin_ctzll(behind);
                t.group = g0 + at;
                t.row0 = lane_value(lo, at) + (place_in - __builtin_amdgcn_readlane(upto[0] - count, at)) * kFewRows;
                behind_last = lane_value(hi, at);
                found = true;
            }
            run_up = __builtin_amdgcn_readlane(upto[0], 63);
        }
        if (!found) return;
        t.rows = (int32_t)min(behind_last - t.row0, (int64_t)kFewRows);
        t.n0 = (int32_t)(w % nlow) * LOW;
        product_tile<FMT, GATED, kLowColumns, kFewRows / 32>(a, t, smem, tid);
        __syncthreads();                           // every wave's results have left LDS
    }
}

template <int FMT, bool GATED, int FW>
__global__ __launch_bounds__(kThreads, 1) void product_tile_kernel(ProductArgs a, int32_t height, int64_t first, int64_t launched) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[kTileLds];
    constexpr int SIDES = GATED ? 2 : 1, COLS = 32 * FW / SIDES, LOW = 32 * kLowColumns / SIDES;
    static_assert(FW >= kLowColumns, "columns of a low tile");
    const int32_t nt = (a.N + COLS - 1) / COLS, nlow = (a.N + LOW - 1) / LOW;
    // One tile a workgroup: the next one starts wherever a CU is done first.  (No loop over tiles: what the compiler keeps across
    // one costs registers that a tile needs, and memory to spill them to costs every workgroup its start: 8192 x 4096 x 7168
    // 178 us, without 171.)
    const int tid = threadIdx.x, lane = tid & 63;
    // Every wave finds the tile for itself, in registers: how many row tiles of each class there are, then the group.
    Groups own = {};
    int32_t sums[kClasses] = {}, total[kClasses] = {};
    for (int32_t g0 = 0; g0 < a.G; g0 += 64) {
        own = groups_at(a, g0 + lane, height);
#pragma unroll
        for (int i = 0; i < kClasses; ++i) sums[i] = own.cut.kind == i ? own.cut.count : 0;
        wave_sums(sums);
#pragma unroll
        for (int i = 0; i < kClasses; ++i) total[i] += __builtin_amdgcn_readlane(sums[i], 63);
    }
    int64_t all = 0;
#pragma unroll
    for (int i = 0; i < kClasses; ++i) all += (int64_t)total[i] * (i == kFew ? nlow : nt);
    // Workgroup b runs on XCD b mod 8.  Of every 256 tiles in the list an XCD has 32 neighbours, which share rows of x and of the weights
    // in its L2; every other 256 in reverse, since tiles are listed by height: the XCDs that had the lowest ones take the next first.
    // Tiles of one group are alike: fewer than 256 at the end are spread over all XCDs.
    const int64_t block = first + blockIdx.x, round = block / 256;
    // Only groups that overlap, where offsets fall, can have more tiles than there are workgroups in all launches.
    if (__builtin_expect(all > launched, 0)) {
        overlapping_tiles<FMT, GATED>(smem, tid, block, launched);
        return;
    }
    const int32_t left = (int32_t)min(all - round * 256, (int64_t)256), run = a.G == 1 ? (left + 7) / 8 : 32;
    const int32_t xcd = (int32_t)(block % 8), in_run = (int32_t)(block % 256 / 8), in_round = (round & 1 ? 7 - xcd : xcd) * run + in_run;
    if (in_run >= run || in_round >= left) return;
    const int64_t w = round * 256 + in_round;
    int64_t begin = 0;
    int kind = kClasses;
#pragma unroll
    for (int i = 0; i < kClasses; ++i)
        if (kind == kClasses) {
            const int64_t tiles = (int64_t)total[i] * (i == kFew ? nlow : nt);
            if (w < begin + tiles) kind = i;
            else begin += tiles;
        }
    const uint32_t columns = (uint32_t)(kind == kFew ? nlow : nt);
    const int64_t in_class = w - begin;
    // (a list of 2^32 tiles and more is one that nobody waits for)
    const int32_t place_in = in_class >> 32 ? (int32_t)(in_class / columns) : (int32_t)((uint32_t)in_class / columns);
    Tile t = {};
    int32_t before = 0, height_in = 0, count_in = 0;
    int64_t lo = 0, hi = 0;
    for (int32_t g0 = 0, run_up = 0;; g0 += 64) {
        int32_t upto[1] = {0};
        if (a.G > 64) {
            own = groups_at(a, g0 + lane, height);
            upto[0] = own.cut.kind == kind ? own.cut.count : 0;
            wave_sums(upto);
        } else {
#pragma unroll
            for (int i = 0; i < kClasses; ++i)
                if (kind == i) upto[0] = sums[i];
        }
        upto[0] += run_up;
        const uint64_t behind = __ballot(upto[0] > place_in);
        if (behind) {
            const int at = __builtin_ctzll(behind);
            t.group = g0 + at;
            height_in = __builtin_amdgcn_readlane(own.cut.height, at);
            count_in = __builtin_amdgcn_readlane(own.cut.count, at);
            before = __builtin_amdgcn_readlane(upto[0], at) - count_in;
            lo = lane_value(own.lo, at);
            hi = lane_value(own.hi, at);
            break;
        }
        run_up = __builtin_amdgcn_readlane(upto[0], 63);
    }
    int32_t tr, tc;
    place((uint32_t)(in_class - (int64_t)before * columns), (uint32_t)count_in, columns, tr, tc);
    t.row0 = lo + (int64_t)tr * height_in;
    t.rows = (int32_t)min((int64_t)height_in, hi - t.row0);
    t.n0 = tc * (kind == kFew ? LOW : COLS);
    if (kind == kFew) {
        if (t.rows > 32) product_tile<FMT, GATED, kLowColumns, 2>(a, t, smem, tid);
        else product_tile<FMT, GATED, kLowColumns, 1>(a, t, smem, tid);
    } else if constexpr (FW == 8) {
        if (t.rows > 224) product_tile<FMT, GATED, FW, 8>(a, t, smem, tid);
        else if (t.rows > 192) product_tile<FMT, GATED, FW, 7>(a, t, smem, tid);
        else if (t.rows > 160) product_tile<FMT, GATED, FW, 6>(a, t, smem, tid);
        else if (t.rows > 128) product_tile<FMT, GATED, FW, 5>(a, t, smem, tid);
        else if (t.rows > 64) product_tile<FMT, GATED, FW, 4>(a, t, smem, tid);
        else product_tile<FMT, GATED, FW, 2>(a, t, smem, tid);
    } else {
        if (t.rows > 64) product_tile<FMT, GATED, FW, 4>(a, t, smem, tid);
        else product_tile<FMT, GATED, FW, 2>(a, t, smem, tid);
    }
}

template <int FMT, bool GATED, int FW> hipError_t launch_width(const ProductArgs &a, int32_t height, hipStream_t s) {
    constexpr int SIDES = GATED ? 2 : 1, COLS = 32 * FW / SIDES, LOW = 32 * kLowColumns / SIDES;
    const int64_t nt = (a.N + COLS - 1) / COLS, nlow = (a.N + LOW - 1) / LOW;
    // Most tiles that groups without common rows can have.  (Heights round up to whole fragments: that leaves out tiles, never adds one.)
    const int64_t tiles = (a.M / height + std::min<int64_t>(a.M / (kFewRows + 1), a.G)) * nt + std::min<int64_t>(a.M, a.G) * nlow;
    const int64_t launched = (tiles + 255) / 256 * 256;
    constexpr int64_t MOST = 1 << 22;              // workgroups of a launch, which has fewer than 2^32 threads
    for (int64_t first = 0; first < tiles; first += MOST) {
        const int64_t grid = (std::min(tiles - first, MOST) + 255) / 256 * 256;
        hipLaunchKernelGGL((product_tile_kernel<FMT, GATED, FW>), dim3((unsigned)grid), dim3(kThreads), 0, s, a, height, first, launched);
    }
    return hipGetLastError();
}
template <int FMT> hipError_t launch_tiles(const ProductArgs &a, int32_t width, int32_t height, hipStream_t s) {
    if (width == 256) return a.up ? launch_width<FMT, true, 8>(a, height, s) : launch_width<FMT, false, 8>(a, height, s);
    return a.up ? launch_width<FMT, true, 4>(a, height, s) : launch_width<FMT, false, 4>(a, height, s);
}

}  // namespace
}  // namespace craft
