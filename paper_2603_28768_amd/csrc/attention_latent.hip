// Attention of one new token per request over a cache of latent rows: up to 576 elements a token, the first 512 of
// them its value row too, shared by all query heads (or a few groups of them).
//
// The products, their operands and the softmax are those of attention.hip (out^T = V^T P^T, S^T = K Q^T, weights
// used where the first product leaves them).  What is different is the ratio: 128 heads make 2 (576 + 512) 128
// operations of 1152 bytes, more than the matrix units' share of what HBM delivers, so every row is fetched once
// for many heads, into LDS.  From there K is read as rows and V by columns, by each of the waves that hold the
// heads.
//
// A workgroup holds 64 heads, 16 a wave, one wave per SIMD unit: Q, the sums of 512 columns and what is on its way
// from LDS take more than half of a SIMD unit's registers.  The products of a tile's scores run before those of the
// tile in front of it with its values, so that the softmax of the one hides behind the other.  Rows travel straight
// into LDS, up to three tiles of 32 tokens ahead, 16-byte pieces in an order (exclusive or with the row's number) in
// which neither way of reading meets a bank twice.  Rows that a tile lacks (behind the last
// token, in front of the window, without a page) are fetched from a row of zeros and masked by -infinity.
//
// Weights are rounded to bf16, the operand's type, in front of the second product: off by 2^-8 of themselves at most.  As two
// bf16 numbers, which attention.hip uses, they would need as many products again, here where the products count: 64
// requests of 1000 to 8000 tokens, 128 heads, 104 us would be 120, 7 of 20000 to 50000 in 8 bits 127 would be 140, and the
// largest errors, at values of 2 to 4, 0.0078 and 0.0151 (the result's own rounding), not 0.0114 and 0.0208.
//
// 64 requests of 1000 to 8000 tokens, 128 heads, bf16: 107 us, 2.5 TB/s and 560 TFLOP/s; 7 of 20000 to 50000 in 8 bits 127
// us, 500 TFLOP/s.  A tile of 32 tokens takes a workgroup 1.3 us (8 bits 1.8), 1.0 of them without any row fetched, and
// 0.45 its 68 matrix instructions.  Reads of a tile out of LDS, by four waves, take 0.9 at 128 bytes a clock; but with 32
// heads a wave, which halves them (and what is widened in 8 bits) for a head and takes all registers, the first takes 134
// us and the second 137.
#include <algorithm>

#include "attention_common.h"

namespace craft {
namespace {

// What an item costs beside its units: queries, first rows, results, 10 us when every CU does it at once.  200 requests
// of 200 to 2500 tokens, 64 heads, with 4 / 6 / 8 / 10: 82.5 / 78 / 76 / 77.5 us.
constexpr int kItemCost = 8;
// Of a workgroup, where there is little to do.  With 4 / 6 / 8 / 12, 128 heads: one request of 900 tokens 18.5 / 19.7 / 22.8 / 24.8 us, 8
// of 600 22.1 / 23.7 / 26.0 / 30.0; 3 of 5000 to 50000 in 8 bits, 32 heads, 37.8 / 37.8 / 37.0 / 41.2; longer ones do not come to it.
constexpr int kMinRun = 6;

// Whether there are fewer items than runs: every item then has a place among the cuts, otherwise every run has (it
// leaves at most one item open).  The join has a workgroup or more for each place.
__host__ __device__ __forceinline__ bool cuts_by_item(const AttentionArgs &a) { return (int64_t)a.R * a.heads <= a.workers; }

__device__ const uint4 zero_row[72] = {};          // 1152 bytes

// dma_chunk (16 bytes a lane) and the same of 4 bytes a lane, by the lanes of a mask, between instructions that all
// lanes run: no branch parts the products.
static __device__ __forceinline__ void dma_chunk_by(uint64_t lanes, ubase_t base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1"
                 :: "s"(lds), "v"(off), "s"(base), "s"(lanes) : "memory");
}
static __device__ __forceinline__ void dma_word_by(uint64_t lanes, ubase_t base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b64 exec, -1"
                 :: "s"(lds), "v"(off), "s"(base), "s"(lanes) : "memory");
}
// from an address of each lane's own
static __device__ __forceinline__ void dma_word_at(ubase_t p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(lds), "v"(p) : "memory");
}
static __device__ __forceinline__ void dma_chunk_at(ubase_t p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(p) : "memory");
}

// Where a row's 16-byte pieces lie: piece p in place p ^ place_of(row), so that what LDS delivers in a clock, 256
// bytes, lies in 64 banks: a read of keys takes a piece of rows 0 to 3 and 12 to 15 and the next one of rows 4 to
// 11, or the other way round; a transposed read of values two neighbouring pieces of rows 0 to 7 or 8 to 15, or (8
// bits) one piece of these rows of either tile of a unit.
template <int FMT> __device__ __forceinline__ int place_of(int row) {
    return ((row ^ (row >> 1 & 4)) & 7) << 1 | ((row >> 3 ^ (FMT == CRAFT_KV_E4M3 ? row >> 4 : 0)) & 1);
}
// the same for what lies behind the value part: 128 bytes, or 64
template <int FMT> __device__ __forceinline__ int rest_place_of(int row) { return FMT == CRAFT_KV_BF16 ? row >> 1 & 7 : row >> 2 & 3; }
// The same value, but nothing computed from it is kept from one tile to the next: registers.
__device__ __forceinline__ uint32_t anew(uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
}
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef const u32x4_t __attribute__((address_space(3))) *lds_piece_t;
typedef s16x4_t __attribute__((address_space(3))) *lds_s16x4_t;
typedef i32x2_t __attribute__((address_space(3))) *lds_i32x2_t;

constexpr int kWaves = 4;                          // of a workgroup, 16 heads each
constexpr int kBuffers = 4;                        // tiles in LDS, and on their way there
constexpr int kAhead = 3;                          // steps that reads of LDS are ahead
constexpr int kStep = 2;                           // tiles of 16 columns of a step
typedef Sums<32, 1, false> State;                  // 32 tiles of 16 columns

// FMT: CRAFT_KV_BF16 or CRAFT_KV_E4M3 (codes stay codes in LDS and are widened in front of the products).
template <int FMT>
__global__ __launch_bounds__(64 * kWaves, 1) void latent_kernel(AttentionArgs a, int32_t blocks) {
    typedef Shape<FMT, 576, 512> S;
    constexpr int T = kUnit, RPW = T / kWaves;                       // rows of a tile, rows a wave fetches
    constexpr int RB = 512 * S::B, TB = 64 * S::B;                   // bytes of a row's value part and of the rest
    constexpr int BUF = T * (RB + TB);
    constexpr int kRows = FMT == CRAFT_KV_BF16 ? 1 : 2, kLanes = 64 / kRows;        // rows of a request, lanes of a row
    constexpr int kRequests = FMT == CRAFT_KV_BF16 ? RPW + 1 : RPW / 2 + 2;   // of a wave for a tile
    __shared__ __attribute__((aligned(1024))) unsigned char s_rows[kBuffers * BUF];
    __shared__ __attribute__((aligned(16))) float s_mask[kBuffers][T], s_scale[kBuffers][FMT == CRAFT_KV_E4M3 ? T : 4];
    static_assert(RPW == 8, "a wave fetches eight rows");
    static_assert(kWaves * 16 * 1024 <= sizeof(s_rows), "the results of all waves fit in the buffers");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int32_t worker = blockIdx.x % a.workers, block = blockIdx.x / a.workers;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)s_rows;
    const uint32_t scale0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)&s_scale[0][0];
    Runs runs;
    const Start st = find_start<kWaves, 1>(a, a.heads, kItemCost, a.workers, kMinRun, worker, runs);
    if (tid == 0 && block == 0 && !cuts_by_item(a)) a.cuts[worker].request = -1;
    if (worker >= runs.n) return;
    const int32_t pieces = a.dk / (16 / S::B);     // of a row, 16 bytes each
    int64_t at = runs.start(worker), before = st.before;
    const int64_t end = runs.start(worker + 1);
    int32_t r = st.request, len = st.len;
    const int32_t head_in_group = (block * kWaves + wave) * 16, n_heads = min(16, a.group - head_in_group);
    State z;
    // where this lane's pieces of eight whole rows lie: of the first row (or two) of the value part, and of the rest
    const bool whole_rows = a.shift >= 3 && pieces == 72 / kRows;
    const uint32_t main_row = FMT == CRAFT_KV_BF16 ? 0u : (uint32_t)(lane >> 5) * (uint32_t)a.k_token;
    const uint32_t main_off = (uint32_t)((lane & (kLanes - 1)) ^ place_of<FMT>(wave * RPW + (FMT == CRAFT_KV_BF16 ? 0 : lane >> 5))) * 16;
    const int in_rest = FMT == CRAFT_KV_BF16 ? lane >> 3 : lane >> 2 & (RPW - 1);
    const uint32_t rest_off = (uint32_t)in_rest * (uint32_t)a.k_token + (kLanes + ((lane & (FMT == CRAFT_KV_BF16 ? 7 : 3)) ^ rest_place_of<FMT>(wave * RPW + in_rest))) * 16;
    // where this lane reads: its first key piece in the value part of a unit's rows and behind it, and its first
    // value.  Pieces and tiles of columns are read in the order of their places, so that those 256 bytes apart follow
    // one another and share an address.
    const int value_row = FMT == CRAFT_KV_BF16 ? 4 * g + (col >> 2) : (col >> 3) * 16 + 4 * g + (col >> 1 & 3);
    const uint32_t key_at = col * RB + (g ^ place_of<FMT>(col)) * 16, rest_at = col * TB + (g ^ rest_place_of<FMT>(col)) * 16;
    const uint32_t value_at = value_row * RB + ((FMT == CRAFT_KV_BF16 ? col >> 1 & 1 : 0) ^ place_of<FMT>(value_row)) * 16 + (col & 1) * 8;
    constexpr int kRows256 = RB / 256;
    auto key_step = [](int i) { return i < RB / 64 ? i % kRows256 * 4 + i / kRows256 : i; };
    auto value_tile = [](int i) { return i % kRows256 * (32 / kRows256) + i / kRows256; };

    while (at < end) {
        const int32_t first = first_of(a, len), n_units = units_of(a, len), cost = n_units + kItemCost, n = len;
        const int64_t in_request = at - before;
        const int32_t h = in_request >> 32 ? (int32_t)(in_request / cost) : (int32_t)((uint32_t)in_request / (uint32_t)cost);
        const int64_t item_begin = before + (int64_t)h * cost, item_end = item_begin + cost;
        const int64_t stop = min(end, item_end);
        const int32_t u0 = max(0, (int32_t)(at - item_begin) - kItemCost), u1 = max(0, (int32_t)(stop - item_begin) - kItemCost);
        const int32_t request = r;
        at = stop;
        if (at == before + (int64_t)cost * a.heads && at < end) {
            before = at;
            ++r;
            len = uniform(length_of(a, r));
        }
        if (u0 == u1) continue;
        const int32_t token0 = (first / kUnit + u0) * kUnit, token1 = min(n, (first / kUnit + u1) * kUnit);

        // ---- a tile into LDS: this wave's rows.  Lane i has the place of row i of them.
        const unsigned char *kh = a.k + h * a.k_head;
        const int32_t *table = a.table + (int64_t)request * a.table_stride;
        const int32_t in_page = (1 << a.shift) - 1;
        auto entry = [&](int32_t i) -> int32_t { return table[min(i, a.max_pages - 1)]; };
        int32_t held0 = (token0 + wave * RPW) >> a.shift;
        int32_t held = entry(held0 + lane), behind = entry(held0 + 64 + lane);
        // A tile's requests go out one by one between the products, since a wave waits where it asks for more than the
        // memory pipeline takes at once.  That is for eight whole rows of one page, which share an address; what else
        // there is (rows that are not there, short rows, small pages) is asked for when it is planned.  Tiles behind
        // the last one are asked for as well (as zeros), so that there are always as many requests on their way.
        bool later = false;                        // the planned requests are still to be made
        ubase_t from = nullptr, from_scale = nullptr;
        uint32_t to_main = 0, to_rest = 0, to_scale = 0;
        auto plan = [&](int32_t tile, int b) __attribute__((always_inline)) {
            const int32_t t0 = token0 + tile * T + wave * RPW;
            // A wave's eight rows begin a page, or lie in one, or begin a whole number of pages (t0 is a multiple of
            // eight): they never lie on either side of the 64 entries held.
            if ((t0 >> a.shift) - held0 >= 64) {
                held0 += 64;
                held = behind;
                behind = entry(held0 + 64 + lane);
            }
            to_main = lds0 + b * BUF + wave * RPW * RB;
            to_rest = lds0 + b * BUF + T * RB + wave * RPW * TB;
            to_scale = scale0 + (b * T + wave * RPW) * 4;
            const int32_t page0 = __builtin_amdgcn_readlane(held, ((t0 >> a.shift) - held0) & 63);
            later = whole_rows && t0 >= first && t0 + RPW <= token1 && (uint32_t)page0 < (uint64_t)a.pages;
            if (later) {
                from = kh + page0 * a.k_page + (t0 & in_page) * a.k_token;
                if (FMT == CRAFT_KV_E4M3) from_scale = reinterpret_cast<ubase_t>(a.k_scale + ((((int64_t)page0 * a.heads + h) << a.shift) + (t0 & in_page)));
                if (lane < RPW) s_mask[b][wave * RPW + lane] = 0.0f;
                return;
            }
            const int lane = (int)anew(tid & 63), my_row = lane & (RPW - 1);
            const int32_t token = t0 + my_row;
            const int32_t page = __shfl(held, ((token >> a.shift) - held0) & 63, 64);
            const bool there = token >= first && token < token1 && (uint32_t)page < (uint64_t)a.pages;
            const unsigned char *row = there ? kh + page * a.k_page + (token & in_page) * a.k_token : reinterpret_cast<const unsigned char *>(zero_row);
            if (lane < RPW) s_mask[b][wave * RPW + lane] = there ? 0.0f : -INFINITY;
            const uint32_t lo = (uint32_t)(uintptr_t)row, hi = (uint32_t)((uintptr_t)row >> 32);
            // what a row lacks at its end is zeros
            auto piece_at = [&](int from, int piece) {
                const ubase_t base = reinterpret_cast<ubase_t>((uint64_t)(uint32_t)__shfl((int)hi, from, 64) << 32 | (uint32_t)__shfl((int)lo, from, 64));
                return (piece < pieces ? base : reinterpret_cast<ubase_t>(zero_row)) + piece * 16;
            };
            const int rest_row = FMT == CRAFT_KV_BF16 ? lane >> 3 : lane >> 2 & (RPW - 1);
            const int rest_piece = kLanes + ((lane & (FMT == CRAFT_KV_BF16 ? 7 : 3)) ^ rest_place_of<FMT>(wave * RPW + rest_row));
            const ubase_t rest = piece_at(rest_row, rest_piece);
            if (FMT == CRAFT_KV_BF16 || lane < 4 * RPW) dma_chunk_at(rest, to_rest);
#pragma unroll
            for (int i = 0; i < RPW; i += kRows) {
                const int in = FMT == CRAFT_KV_BF16 ? 0 : lane >> 5;
                dma_chunk_at(piece_at(i + in, (lane & (kLanes - 1)) ^ place_of<FMT>(wave * RPW + i + in)), to_main + i * RB);
            }
            if (FMT == CRAFT_KV_E4M3) {
                const float *scale = there ? a.k_scale + ((((int64_t)page * a.heads + h) << a.shift) + (token & in_page)) : reinterpret_cast<const float *>(zero_row);
                if (lane < RPW) dma_word_at(reinterpret_cast<ubase_t>(scale), to_scale);
            }
        };
        // request i of the planned ones, if they are still to be made
        auto ask = [&](int i) __attribute__((always_inline)) {
            const uint64_t all = later ? ~0ull : 0ull;
            if (i < RPW / kRows) {
                // the place of row 8 w + i is that of row 8 w and 2 i, exclusive or
                dma_chunk_by(all, from + (uint32_t)(i * kRows) * (uint32_t)a.k_token, (main_off ^ (uint32_t)(i * kRows * 32)) + main_row, to_main + i * kRows * RB);
            } else if (i == RPW / kRows) {
                dma_chunk_by(FMT == CRAFT_KV_BF16 ? all : all & ((1ull << 4 * RPW) - 1), from, rest_off, to_rest);
            } else if (i < kRequests) {
                dma_word_by(all & ((1ull << RPW) - 1), from_scale, lane * 4, to_scale);
            }
        };

        // ---- queries
        u32x4_t q[S::QN];
        {
            const bool live = col < n_heads;
            const __amdgpu_buffer_rsrc_t qr = rows_of(static_cast<const unsigned char *>(a.q) + ((int64_t)request * a.q_stride + (int64_t)(h * a.group + head_in_group) * a.q_head) * 2, kFar);
            const uint32_t q_off = (uint32_t)col * (uint32_t)a.q_head * 2;
#pragma unroll
            for (int i = 0; i < S::QN; ++i) {
                const int d = FMT == CRAFT_KV_E4M3 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 32 + g * 8;
                q[i] = __builtin_amdgcn_raw_buffer_load_b128(qr, live && d < a.dk ? q_off + d * 2 : kFar, 0, 0);
            }
        }
        z.clear();
        // here, and not inside the loop, the compiler waits for them; it knows nothing of the rows on their way, and a
        // wait of its own would wait for those too
#pragma unroll
        for (int i = 0; i < S::QN; ++i) asm volatile("" : "+v"(q[i]));

        constexpr int kEvery = FMT == CRAFT_KV_BF16 ? 4 : 2, kBehindScores = (S::NK + kEvery - 1) / kEvery;
        static_assert(kBehindScores + 4 >= kRequests, "every request goes out behind some products");
        const int32_t tiles = u1 - u0;
        const bool busy = n_heads > 0;
        // every wave's part of a tile has landed, and everybody is done with the tile before the last one
        auto meet = [&]() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
        f32x4_t s[2];
        auto scores = [&](int b, bool more) __attribute__((always_inline)) {
            const uint32_t rows = lds0 + b * BUF, rest = rows + T * RB;
            // a piece's place in its 256 bytes is exclusive-or'ed into the address of the lane's first one
            const uint32_t key0 = anew(rows + key_at), key1 = FMT == CRAFT_KV_E4M3 ? key0 ^ 16 : key0, rest0 = anew(rest + rest_at);
            u32x4_t kr[kAhead + 1][2];
            auto read_keys = [&](int i) __attribute__((always_inline)) {
                const int step = key_step(i);
                if (step < RB / 64) {
                    kr[i % (kAhead + 1)][0] = *(lds_piece_t)(uintptr_t)((key0 ^ (step & 3) * 64) + (step >> 2) * 256);
                    kr[i % (kAhead + 1)][1] = *(lds_piece_t)(uintptr_t)((key1 ^ (step & 3) * 64) + (step >> 2) * 256 + 16 * RB);
                } else {
                    kr[i % (kAhead + 1)][0] = *(lds_piece_t)(uintptr_t)(rest0 ^ (step & 1 & TB / 128) * 64);
                    kr[i % (kAhead + 1)][1] = *(lds_piece_t)(uintptr_t)((rest0 ^ (step & 1 & TB / 128) * 64) + 16 * TB);
                }
            };
            s[0] = s[1] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read_keys(i);
#pragma unroll
            for (int i = 0; i < S::NK; ++i) {
                if (i + kAhead < S::NK) read_keys(i + kAhead);
#pragma unroll
                for (int e = 0; e < (FMT == CRAFT_KV_E4M3 ? 2 : 1); ++e)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const u32x4_t kc = kr[i % (kAhead + 1)][t];
                        const bf16x8_t kf = FMT == CRAFT_KV_BF16 ? __builtin_bit_cast(bf16x8_t, kc) : widen((u32x2_t){kc[2 * e], kc[2 * e + 1]});
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8_t, q[FMT == CRAFT_KV_E4M3 ? 2 * key_step(i) + e : key_step(i)]), s[t], 0, 0, 0);
                    }
                if (more && i % kEvery == 0) ask(i / kEvery);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // The weights of the scores.  What the maximum's growth multiplies the sums by is left to the caller, behind
        // the products that come first; only the sum of the weights has it already.
        float factor = 1.0f;
        auto weights = [&](int b) __attribute__((always_inline)) -> bf16x8_t {
            f32x4_t scale[2];
            float x[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const f32x4_t mask = *reinterpret_cast<const f32x4_t *>(&s_mask[b][t * 16 + 4 * g]);
                if (FMT == CRAFT_KV_E4M3) scale[t] = *reinterpret_cast<const f32x4_t *>(&s_scale[b][t * 16 + 4 * g]);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[t][j] = s[t][j] * (FMT == CRAFT_KV_E4M3 ? a.scale_log2 * scale[t][j] : a.scale_log2) + mask[j];
            }
            const float top = max_of_head(fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3]))));
            const float up = top > z.m + kSlack ? top : z.m;
            factor = up == z.m ? 1.0f : __builtin_amdgcn_exp2f(z.m - up);
            z.m = up;
            z.l *= factor;
            const float base = up == -INFINITY ? 0.0f : up;
            float p[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[t][j] = __builtin_amdgcn_exp2f(x[t][j] - base);
                    z.l += p[t][j];
                    if (FMT == CRAFT_KV_E4M3) p[t][j] *= scale[t][j];
                }
            const wide_t pw = {bf16_pair(p[0][0], p[0][1]), bf16_pair(p[0][2], p[0][3]), bf16_pair(p[1][0], p[1][1]), bf16_pair(p[1][2], p[1][3])};
            return __builtin_bit_cast(bf16x8_t, pw);
        };
        // Values: columns of 16 out of LDS, transposed on the way (a lane gets four, or eight, tokens of its column
        // out of the 8 bytes each that 16 lanes ask for).
        auto values = [&](int b, bf16x8_t pf, bool more) __attribute__((always_inline)) {
            bf16x8_t vf[kAhead + 1][kStep];
            const uint32_t value0 = anew(lds0 + b * BUF + value_at);
            auto read_values = [&](int step) __attribute__((always_inline)) {
#pragma unroll
                for (int c = 0; c < kStep; ++c) {
                    const int tile = value_tile(step * kStep + c);
                    const uint32_t p = (value0 ^ (uint32_t)(tile % (256 / (16 * S::B))) * (16 * S::B)) + tile / (256 / (16 * S::B)) * 256;
                    if (FMT == CRAFT_KV_BF16) {
                        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(uintptr_t)p);
                        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(uintptr_t)(p + 16 * RB));
                        vf[step % (kAhead + 1)][c] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    } else {
                        vf[step % (kAhead + 1)][c] = widen(__builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_t)(uintptr_t)p)));
                    }
                }
            };
#pragma unroll
            for (int i = 0; i < kAhead; ++i) read_values(i);
#pragma unroll
            for (int i = 0; i < 32 / kStep; ++i) {
                if (i + kAhead < 32 / kStep) read_values(i + kAhead);
#pragma unroll
                for (int c = 0; c < kStep; ++c)
                    z.acc[value_tile(i * kStep + c)][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[i % (kAhead + 1)][c], pf, z.acc[value_tile(i * kStep + c)][0], 0, 0, 0);
                if (more && i % 4 == 1) ask(kBehindScores + i / 4);
            }
        };
        auto rescale = [&]() __attribute__((always_inline)) {
            if (__any(factor != 1.0f)) {
#pragma unroll
                for (int c = 0; c < 32; ++c) z.acc[c][0] *= factor;
            }
        };

        for (int i = 0; i < kBuffers - 1; ++i) {
            plan(i, i);
#pragma unroll
            for (int j = 0; j < kRequests; ++j) ask(j);
        }
        dma_wait<2 * kRequests>();
        meet();
        bf16x8_t pf = {};
        if (busy) {
            scores(0, false);
            pf = weights(0);
        }
        for (int32_t tile = 0; tile + 1 < tiles; ++tile) {
            dma_wait<kRequests>();
            meet();
            const int next = (tile + 3) % kBuffers;
            plan(tile + 3, next);
            if (busy) {
                scores((tile + 1) % kBuffers, true);
                const bf16x8_t pn = weights((tile + 1) % kBuffers);
                values(tile % kBuffers, pf, true);
                rescale();
                pf = pn;
            } else {
#pragma unroll
                for (int j = 0; j < kRequests; ++j) ask(j);
            }
        }
        if (busy) values((tiles - 1) % kBuffers, pf, false);
        dma_wait<0>();
        meet();                                    // the buffers are free for the next item

        // Results leave as whole rows, by way of the buffers: piece p of 16 bytes of a head's row in place p ^ head.
        // Straight out of the registers a store instruction has 32 bytes of each of 16 rows: 7900 cycles an item, not 4600.
        auto write_rows = [&](int32_t to, int32_t head0) {
            unsigned char *rows = s_rows + wave * 16 * 1024;
            const float sum = sum_of_head(z.l), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                const f32x4_t x = z.acc[c][0] * inv;
                *reinterpret_cast<u32x2_t *>(rows + col * 1024 + ((c * 2 + (g >> 1)) ^ col) * 16 + (g & 1) * 8) = (u32x2_t){bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
            }
            const int64_t head = (int64_t)to * a.Hq + head0;
            if (a.lse && g == 0 && col < n_heads) a.lse[head + col] = sum == 0.0f ? -INFINITY : (z.m + __log2f(sum)) * 0.6931471805599453f;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            unsigned char *out = static_cast<unsigned char *>(a.out) + (head * a.dv + lane * 8) * 2;
            for (int i = 0; i < n_heads; ++i) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t *>(rows + i * 1024 + (lane ^ i) * 16);
                if (lane * 8 < a.dv) *reinterpret_cast<u32x4_t *>(out + (int64_t)i * a.dv * 2) = x;
            }
        };
        const bool starts = u0 == 0, ends = u1 == n_units;
        if (busy) {
            if (starts && ends) write_rows(request, h * a.group + head_in_group);
            else z.put(a.part + (((int64_t)worker * 2 + (starts ? 1 : 0)) * blocks * kWaves + block * kWaves + wave) * State::kFloats, lane);
        }
        if (starts && ends) meet();                // the buffers are free again
        if (starts && tid == 0 && block == 0 && (!ends || cuts_by_item(a)))
            a.cuts[cuts_by_item(a) ? request * a.heads + h : worker] = {ends ? -1 : request, h, worker, ends ? 0 : runs.of(item_end - 1)};
    }
}

// Joins the parts of the items that are cut between workgroups: the last part of the run that an item starts in and the
// first ones of those that follow.  A launch of its own, because the parts are many (33 KiB for every 16 heads) and
// their sum wants many CUs: a workgroup has TILES tiles of columns of 16 heads, its waves every fourth part.
template <int TILES>
__global__ __launch_bounds__(64 * kWaves) void latent_join_kernel(AttentionArgs a, int32_t blocks) {
    typedef Sums<TILES, 1, false> Some;
    constexpr int kColumns = 32 / TILES;           // workgroups of a set
    __shared__ float s_sums[kWaves][Some::kFloats];
    const int32_t set = blockIdx.y / kColumns;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tile0 = blockIdx.y % kColumns * TILES;
    const LatentCut cut = a.cuts[blockIdx.x];
    const int32_t run = cut.first;
    const int32_t n_heads = min(16, a.group - set * 16);
    if (cut.request < 0 || n_heads <= 0 || tile0 * 16 >= a.dv) return;
    Some z;
    z.clear();
#pragma unroll 2
    for (int32_t w = run + wave; w <= cut.last; w += kWaves) {
        const float *part = a.part + (((int64_t)w * 2 + (w == run ? 1 : 0)) * blocks * kWaves + set) * State::kFloats;
        z.join(part[State::kFloats - 128 + lane], part[State::kFloats - 64 + lane],
               [&](int c, int) { return *reinterpret_cast<const f32x4_t *>(part + ((tile0 + c) * 64 + lane) * 4); });
    }
    if (wave > 0) z.put(s_sums[wave], lane);
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kWaves && run + w <= cut.last; ++w) z.add(s_sums[w], lane);
    z.write(a, cut.request, cut.head * a.group + set * 16, n_heads, lane, tile0);
}

int32_t latent_blocks(const AttentionArgs &a) { return (a.group + 16 * kWaves - 1) / (16 * kWaves); }

template <int FMT>
void launch_format(const AttentionArgs &a, hipStream_t s) {
    const int32_t blocks = latent_blocks(a);
    hipLaunchKernelGGL((latent_kernel<FMT>), dim3((unsigned)(a.workers * blocks)), dim3(64 * kWaves), 0, s, a, blocks);
    const int32_t cuts = cuts_by_item(a) ? a.R * a.heads : a.workers;
    // Items of many parts have few workgroups at four tiles each: 3 of 5000 to 50000 tokens in 8 bits, 32 heads, 48.5 us, at two
    // tiles 38; 30 of 500 to 20000, 16 heads, 52.6 and 50.6.  Items of few parts have enough: 64 of 1000 to 8000, 128 heads,
    // 110 us at four, 112 at two.
    if (cuts * 8 <= a.workers) hipLaunchKernelGGL(latent_join_kernel<2>, dim3((unsigned)cuts, (unsigned)(blocks * kWaves * 16)), dim3(64 * kWaves), 0, s, a, blocks);
    else hipLaunchKernelGGL(latent_join_kernel<4>, dim3((unsigned)cuts, (unsigned)(blocks * kWaves * 8)), dim3(64 * kWaves), 0, s, a, blocks);
}

}  // namespace

// A workgroup per CU; those of one run and different heads read the same rows, so they get numbers that meet in one
// XCD (multiples of 8 apart).
int32_t latent_workers(const AttentionArgs &a, int32_t num_cu) {
    const int32_t n = std::max(1, num_cu / latent_blocks(a));
    return n >= 8 ? n / 8 * 8 : n;
}

size_t latent_workspace(const AttentionArgs &a, int32_t num_cu) {
    const size_t w = (size_t)latent_workers(a, num_cu);
    return w * sizeof(LatentCut) + w * 2 * latent_blocks(a) * kWaves * State::kFloats * sizeof(float);
}

hipError_t launch_latent_attention(const AttentionArgs &args, void *workspace, hipStream_t s) {
    AttentionArgs a = args;
    a.cuts = static_cast<LatentCut *>(workspace);
    a.part = reinterpret_cast<float *>(a.cuts + a.workers);
    if (a.format == CRAFT_KV_BF16) launch_format<CRAFT_KV_BF16>(a, s);
    else launch_format<CRAFT_KV_E4M3>(a, s);
    return hipGetLastError();
}

}  // namespace craft
