// Attention of one new token per request over the paged key/value cache.
//
//   s[i] = scale q . K[i],  m = max s,  p[i] = exp(s[i] - m),  out = sum p[i] V[i] / sum p[i]
//
// in one pass over the cache: a wave keeps the running m, l = sum p and acc = sum p V of its tokens, and
// multiplies l and acc by exp(m_old - m_new) when the maximum grows.  Per cached element 2 * group operations
// against 1 to 4 bytes: bound by HBM, the matrix instructions are there because they do the sums over d and
// over tokens without shuffles, whatever the number of heads that share a key.
//
// A unit is 32 tokens of one cache head, two tiles of 16, against up to 16 query heads that share it.  Both
// products have the heads in the columns (lane & 15), so maxima, sums and weights of a head stay in its lanes:
//   S^T = K Q^T     a lane's row of the left operand is a token, its elements 16-byte pieces of that row.  In
//                   which order the contraction over d is summed is free, so the pieces are taken as they lie in
//                   memory (lane >> 4 picks the piece) and Q is laid out alike.
//   out^T = V^T P^T the contraction runs over tokens: in which order is free again, and is chosen so that the
//                   weights are used where the first product leaves them (lane group g holds tokens 4g .. 4g + 3
//                   of either tile).  The row of the left operand is a column of V; which column is free: row
//                   r of tile j is column CE r + j, so that a lane reads CE neighbouring elements of a token,
//                   the 16 lanes of a group a contiguous stretch, and transposes 8 tokens x CE within its own
//                   registers.  No LDS and no shuffle in the loop.
// A wave has the keys of the next unit in flight while it works on the weights and values of this one, and the
// other way round.
//
// Work: the (request, head) items, each its units and a few more for what an item costs by itself, are laid end
// to end and cut into equal runs, one per wave, by prefix sums over the lengths that every workgroup does for
// itself: the launch does not depend on the lengths (which the host does not know), and long and short requests
// take equal parts of the GPU.  A wave walks its run alone; what it begins and does not end, or ends and did not
// begin, meets the neighbouring waves' sums in LDS at the end of the workgroup.  An item cut between workgroups
// leaves partial sums, which a second launch joins in the order of the workgroups.
#include <algorithm>

#include "ffn_common.h"

namespace craft {
namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kUnit = 32;                          // tokens
constexpr int kItemCost = 2;                       // what an item costs beside its units
constexpr int kMinRun = 4;                         // of a wave, where there is little to do
constexpr uint32_t kFar = 0x80000000u;             // an offset behind the end of every page: reads as zeros

// Elements of 16 bytes, of the widest value load of a lane, and what the products take.
template <int FMT> struct Format;
template <> struct Format<CRAFT_KV_F32> { static constexpr int kBytes = 4, kPiece = 4; };
template <> struct Format<CRAFT_KV_BF16> { static constexpr int kBytes = 2, kPiece = 8; };
template <> struct Format<CRAFT_KV_E4M3> { static constexpr int kBytes = 1, kPiece = 16; };

template <int FMT, int DK, int DV> struct Shape {
    static constexpr int B = Format<FMT>::kBytes;
    static constexpr int NK = DK * B / 64;                          // 16-byte key pieces of a lane per tile
    static constexpr int CE = DV / 16 < Format<FMT>::kPiece ? DV / 16 : Format<FMT>::kPiece;   // elements of a value load
    static constexpr int NV = DV / 16 / CE;                         // value loads of a lane per token
    static constexpr int VW = CE * B / 4;                           // words of one
    static constexpr int QN = FMT == CRAFT_KV_E4M3 ? 2 * NK : NK;   // 16-byte pieces of the queries
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const unsigned char *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(p), 0, bytes, 0x00027000);
}
template <int W> struct Words;
template <> struct Words<4> {
    typedef u32x4_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0); }
};
template <> struct Words<2> {
    typedef u32x2_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0); }
};
template <> struct Words<1> {
    typedef uint32_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0); }
};
template <int W> __device__ __forceinline__ uint32_t word(const typename Words<W>::type &x, int i) { return x[i]; }
template <> __device__ __forceinline__ uint32_t word<1>(const uint32_t &x, int) { return x; }

// The same in every lane of the wave: kept in scalar registers.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)(x >> 32)) << 32 | (uint32_t)uniform((int32_t)x));
}

// Reductions over the four lanes that hold a head (lane & 15): lanes 16 and 32 apart change places.
__device__ __forceinline__ float other16(float x) {
    return __shfl_xor(x, 16, 64);
}
__device__ __forceinline__ float other32(float x) {
    return __shfl_xor(x, 32, 64);
}
__device__ __forceinline__ float max_of_head(float x) {
    x = fmaxf(x, other16(x));
    return fmaxf(x, other32(x));
}
__device__ __forceinline__ float sum_of_head(float x) {
    x += other16(x);
    return x + other32(x);
}
__device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

__device__ __forceinline__ int32_t units_of(const AttentionArgs &a, int32_t r, int32_t *first, int32_t *len) {
    const int64_t cap = (int64_t)a.max_pages << a.shift;
    const int32_t n = (int32_t)min((int64_t)max(a.lens[r], 0), cap);
    const int32_t lo = a.window > 0 && n > a.window ? n - a.window : 0;
    *first = lo;
    *len = n;
    // an empty request is one unit without tokens, so that somebody writes its zeros
    return max(1, (int32_t)(((int64_t)n + kUnit - 1) / kUnit) - lo / kUnit);
}

// The list of items cut into n runs.  Lengths in units, an item's own cost included.
struct Runs {
    int64_t total, each;   // the first `more` runs are one longer than `each`
    int32_t n, more;
    __device__ __forceinline__ void cut(int64_t t, int32_t most) {
        total = t;
        n = (int32_t)min((int64_t)most, (t + kMinRun - 1) / kMinRun);
        if (t >> 32) {
            each = t / n;
        } else {
            each = (uint32_t)t / (uint32_t)n;
        }
        more = (int32_t)(t - each * n);
    }
    __device__ __forceinline__ int64_t start(int32_t w) const { return each * w + min(w, more); }
    __device__ __forceinline__ int32_t of(int64_t at) const {      // the run that holds place `at`
        const int64_t longer = (each + 1) * more;
        return at < longer ? (int32_t)(at / (each + 1)) : more + (int32_t)((at - longer) / each);
    }
};

// The request in which each wave's run starts, and the cost in front of it.
struct Start {
    int64_t before;
    int32_t request;
};
// per_request: items of a request (heads x blocks of 16 query heads).
__device__ __forceinline__ Start find_start(const AttentionArgs &a, int32_t per_request, Runs &runs) {
    __shared__ int64_t wave_sum[kWaves];
    __shared__ Start found[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t per = (a.R + kThreads - 1) / kThreads;
    const int64_t r0 = min((int64_t)a.R, (int64_t)tid * per), r1 = min((int64_t)a.R, r0 + per);
    int64_t sum = 0;
    int32_t lo, len;
    for (int64_t r = r0; r < r1; ++r) sum += units_of(a, (int32_t)r, &lo, &len) + kItemCost;
    sum *= per_request;
    int64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t up = __shfl_up(incl, d, 64);
        if (lane >= d) incl += up;
    }
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    int64_t before = incl - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += wave_sum[w];
        total += wave_sum[w];
    }
    runs.cut(uniform(total), a.workers * kWaves);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int32_t rank = blockIdx.x * kWaves + w;
        const int64_t at = runs.start(rank);
        if (rank < runs.n && at >= before && at < before + sum) {
            int64_t b = before;
            int32_t r = (int32_t)r0;
            for (;; ++r) {
                const int64_t u = (int64_t)(units_of(a, r, &lo, &len) + kItemCost) * per_request;
                if (at < b + u) break;
                b += u;
            }
            found[w] = {b, r};
        }
    }
    __syncthreads();
    return {uniform(found[wave].before), uniform(found[wave].request)};
}

// Running maximum, sum of weights and weighted sum of some tokens of an item, as a wave holds them: lane (head, g)
// has the sum of the weights of its own tokens only, the rest is whole.
template <int NV, int CE> struct Sums {
    f32x4_t acc[NV][CE];
    float m, l;
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) acc[c][e] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
    }
    __device__ __forceinline__ void scale(float f) {
        l *= f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) acc[c][e] *= f;
    }
    // Sums in memory: the accumulators, then m, then l, lane by lane.
    static constexpr int kFloats = (NV * CE * 4 + 2) * 64;
    __device__ __forceinline__ void put(float *to, int lane) const {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) *reinterpret_cast<f32x4_t *>(to + ((c * CE + e) * 64 + lane) * 4) = acc[c][e];
        to[NV * CE * 256 + lane] = m;
        to[NV * CE * 256 + 64 + lane] = l;
    }
    __device__ __forceinline__ void add(const float *from, int lane) {
        const float om = from[NV * CE * 256 + lane], ol = from[NV * CE * 256 + 64 + lane];
        const float up = fmaxf(m, om);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - up), of = om == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(om - up);
        m = up;
        l = l * f + ol * of;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t *>(from + ((c * CE + e) * 64 + lane) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[c][e][i] = acc[c][e][i] * f + x[i] * of;
            }
    }
    // Row i of tile (c, e) is column (c 16 + 4 g + i) CE + e: CE neighbouring columns of the output per (c, i).
    template <bool F32> __device__ __forceinline__ void write(const AttentionArgs &a, int32_t r, int32_t head0, int32_t n_heads, int lane) const {
        const int col = lane & 15, g = lane >> 4;
        const float sum = sum_of_head(l);
        if (col >= n_heads) return;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int64_t head = (int64_t)r * a.Hq + head0 + col;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = (c * 16 + 4 * g + i) * CE;
                if (d >= a.dv) continue;
                if constexpr (F32) {
                    *reinterpret_cast<f32x4_t *>(static_cast<float *>(a.out) + head * a.dv + d) =
                        (f32x4_t){acc[c][0][i] * inv, acc[c][1][i] * inv, acc[c][2][i] * inv, acc[c][3][i] * inv};
                } else {
                    uint32_t w[CE / 2];
#pragma unroll
                    for (int e = 0; e < CE / 2; ++e) w[e] = bf16_pair(acc[c][2 * e][i] * inv, acc[c][2 * e + 1][i] * inv);
                    unsigned char *to = static_cast<unsigned char *>(a.out) + (head * a.dv + d) * 2;
                    if constexpr (CE == 4) {
                        *reinterpret_cast<u32x2_t *>(to) = (u32x2_t){w[0], w[1]};
                    } else {
#pragma unroll
                        for (int e = 0; e < CE / 8; ++e) *reinterpret_cast<u32x4_t *>(to + 16 * e) = (u32x4_t){w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]};
                    }
                }
            }
        if (g == 0 && a.lse) a.lse[head] = sum == 0.0f ? -INFINITY : (m + __log2f(sum)) * 0.6931471805599453f;
    }
};

// Pages of the tokens that a lane reads of a unit.  Pages of 16 tokens and more: one for either tile, the same in
// every lane.  SMALL pages: of the lane's key row in either tile, and of the tokens whose values it reads, which
// are those whose scores it holds.  -1: no such token, or no page.
template <bool SMALL> struct Pages { int32_t tile[2]; };
template <> struct Pages<true> { int32_t key[2], value[8]; };

// WPS: workgroups of a CU that the registers must do for.  AHEAD: the next unit's rows are requested while this
// one's are worked on (registers for a whole unit); otherwise a piece is requested where it is used.
template <int FMT, int DK, int DV, bool SMALL, bool AHEAD, int WPS>
__global__ __launch_bounds__(kThreads, WPS) void decode_kernel(AttentionArgs a, int32_t blocks) {
    typedef Shape<FMT, DK, DV> S;
    typedef Words<S::VW> VWords;
    typedef Sums<S::NV, S::CE> State;
    __shared__ float s_sums[kWaves][State::kFloats];   // of the item that a wave's run found begun
    __shared__ int32_t s_found[kWaves];                // whether there is one, and whether it ends in the run
    enum { kNone = 0, kOpen = 1, kEnded = 2 };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int32_t per_request = a.heads * blocks, rank = blockIdx.x * kWaves + wave;
    Runs runs;
    const Start st = find_start(a, per_request, runs);
    if (tid == 0) a.desc[4 * blockIdx.x] = -1;
    if ((int32_t)blockIdx.x * kWaves >= runs.n) return;
    int64_t at = 0, end = 0, before = st.before;
    if (rank < runs.n) {
        at = runs.start(rank);
        end = runs.start(rank + 1);
    }
    int32_t r = st.request;
    if (lane == 0) s_found[wave] = kNone;
    State z;
    bool open = false;                             // the run ends inside an item that starts in it
    int32_t open_item = 0, open_head0 = 0, open_heads = 0;
    int64_t open_end = 0;

    while (at < end) {
        int32_t first, len;
        const int32_t n_units = uniform(units_of(a, r, &first, &len));
        first = uniform(first);
        len = uniform(len);
        const int32_t cost = n_units + kItemCost;
        const int64_t in_request = at - before;
        const int32_t item = in_request >> 32 ? (int32_t)(in_request / cost) : (int32_t)((uint32_t)in_request / (uint32_t)cost);
        const int64_t item_begin = before + (int64_t)item * cost, item_end = item_begin + cost;
        const int64_t stop = min(end, item_end);
        // an item's own cost comes first
        const int32_t u0 = max(0, (int32_t)(at - item_begin) - kItemCost), u1 = max(0, (int32_t)(stop - item_begin) - kItemCost);
        at = stop;
        const int64_t item_before = before;
        const int32_t item_r = r;
        if (at == item_before + (int64_t)cost * per_request) { before = at; ++r; }
        if (u0 == u1) continue;
        const int32_t h = item / blocks, block = item - h * blocks;
        const int32_t head0 = h * a.group + block * 16, n_heads = min(16, a.group - block * 16);
        const int32_t unit_base = first / kUnit;   // of the request's visible tokens

        // ---- queries: the right operand of the first product, laid out as the key pieces are
        u32x4_t q[S::QN];
        {
            const bool live = col < n_heads;
            constexpr int QB = FMT == CRAFT_KV_F32 ? 4 : 2, QE = 16 / QB;     // bytes of an element, elements of a piece
            const unsigned char *qr = static_cast<const unsigned char *>(a.q) + ((int64_t)item_r * a.q_stride + (int64_t)(head0 + (live ? col : 0)) * a.q_head) * QB;
            const u32x4_t none = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < S::QN; ++i) {
                const int d = FMT == CRAFT_KV_E4M3 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 4 * QE + g * QE;
                q[i] = live && d < a.dk ? *reinterpret_cast<const u32x4_t *>(qr + d * QB) : none;
            }
        }

        const unsigned char *kh = a.k + h * a.k_head, *vh = a.v + h * a.v_head;
        const int32_t *table = a.table + (int64_t)item_r * a.table_stride;
        const uint32_t k_span = 16u * (uint32_t)a.k_token, v_span = 16u * (uint32_t)a.v_token;
        const uint32_t k_off = (uint32_t)col * (uint32_t)a.k_token + g * 16;

        z.clear();

        u32x4_t kr[2][AHEAD ? S::NK : 1];
        typename VWords::type vr[8][AHEAD ? S::NV : 1];
        f32x4_t ks[2], vs[2], vs_next[2];

        auto page_of = [&](int32_t token) -> int32_t {
            const int32_t page = token < len ? table[min(token >> a.shift, a.max_pages - 1)] : -1;
            return (uint32_t)page < (uint64_t)a.pages ? page : -1;
        };
        auto pages_of = [&](int32_t u, bool live) -> Pages<SMALL> {
            Pages<SMALL> pg;
            if constexpr (SMALL) {
#pragma unroll
                for (int t = 0; t < 2; ++t) pg.key[t] = live ? page_of(u * kUnit + t * 16 + col) : -1;
#pragma unroll
                for (int j = 0; j < 8; ++j) pg.value[j] = live ? page_of(u * kUnit + (j >> 2) * 16 + 4 * g + (j & 3)) : -1;
            } else {
#pragma unroll
                for (int t = 0; t < 2; ++t) pg.tile[t] = live ? __builtin_amdgcn_readfirstlane(page_of(u * kUnit + t * 16)) : -1;
            }
            return pg;
        };
        const int32_t in_page = (1 << a.shift) - 1;
        auto load_key = [&](int32_t u, const Pages<SMALL> &pg, int t, int i) __attribute__((always_inline)) -> u32x4_t {
            const int32_t token = u * kUnit + t * 16;
            const bool inside = (i * 4 + g) * Format<FMT>::kPiece < a.dk;
            if constexpr (SMALL) {
                const u32x4_t none = {0u, 0u, 0u, 0u};
                const unsigned char *row = kh + pg.key[t] * a.k_page + ((token + col) & in_page) * a.k_token;
                return inside && pg.key[t] >= 0 ? *reinterpret_cast<const u32x4_t *>(row + i * 64 + g * 16) : none;
            } else {
                const bool good = pg.tile[t] >= 0;
                const __amdgpu_buffer_rsrc_t rs = rows_of(kh + (good ? pg.tile[t] * a.k_page + (token & in_page) * a.k_token : 0), good ? k_span : 0u);
                return __builtin_amdgcn_raw_buffer_load_b128(rs, (inside ? k_off : kFar) + i * 64, 0, 0);
            }
        };
        // rows behind the last token (and in front of the window) may hold anything: read as zeros
        auto load_value = [&](int32_t u, const Pages<SMALL> &pg, bool whole, int t, int j, int c) __attribute__((always_inline)) -> typename VWords::type {
            const int32_t token = u * kUnit + t * 16, row = 4 * g + j;
            const bool inside = (whole || (token + row >= first && token + row < len)) && (c * 16 + col) * S::CE < a.dv;
            if constexpr (SMALL) {
                const int32_t page = pg.value[4 * t + j];
                typename VWords::type x = {};
                if (inside && page >= 0)
                    x = *reinterpret_cast<const typename VWords::type *>(vh + page * a.v_page + ((token + row) & in_page) * a.v_token + (c * 16 + col) * (S::CE * S::B));
                return x;
            } else {
                const bool good = pg.tile[t] >= 0;
                const __amdgpu_buffer_rsrc_t rs = rows_of(vh + (good ? pg.tile[t] * a.v_page + (token & in_page) * a.v_token : 0), good ? v_span : 0u);
                return VWords::load(rs, inside ? (uint32_t)row * (uint32_t)a.v_token + (c * 16 + col) * (S::CE * S::B) : kFar);
            }
        };
        auto load_scales = [&](int32_t u, const Pages<SMALL> &pg) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int32_t token = u * kUnit + t * 16;
                if constexpr (SMALL) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int32_t page = pg.value[4 * t + j];
                        const int64_t so = (((int64_t)page * a.heads + h) << a.shift) + ((token + 4 * g + j) & in_page);
                        ks[t][j] = page >= 0 ? a.k_scale[so] : 0.0f;
                        vs_next[t][j] = page >= 0 ? a.v_scale[so] : 0.0f;
                    }
                } else {
                    const bool good = pg.tile[t] >= 0;
                    const int64_t so = good ? (((int64_t)pg.tile[t] * a.heads + h) << a.shift) + (token & in_page) : 0;
                    ks[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                        rows_of(reinterpret_cast<const unsigned char *>(a.k_scale + so), good ? 64u : 0u), g * 16, 0, 0));
                    vs_next[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                        rows_of(reinterpret_cast<const unsigned char *>(a.v_scale + so), good ? 64u : 0u), g * 16, 0, 0));
                }
            }
        };
        auto load_keys = [&](int32_t u, const Pages<SMALL> &pg) __attribute__((always_inline)) {
            if constexpr (AHEAD) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < S::NK; ++i) kr[t][i] = load_key(u, pg, t, i);
            }
            if (FMT == CRAFT_KV_E4M3) load_scales(u, pg);
        };
        auto all_seen = [&](int32_t u) { return u * kUnit >= first && u * kUnit + kUnit <= len; };
        auto load_values = [&](int32_t u, const Pages<SMALL> &pg) __attribute__((always_inline)) {
            if constexpr (AHEAD) {
                const bool whole = all_seen(u);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int c = 0; c < S::NV; ++c) vr[4 * t + j][c] = load_value(u, pg, whole, t, j, c);
            }
        };

        Pages<SMALL> pages = {};
        if (u0 < u1) {
            pages = pages_of(unit_base + u0, true);
            load_keys(unit_base + u0, pages);
            load_values(unit_base + u0, pages);
        }
        for (int32_t i = u0; i < u1; ++i) {
            const int32_t u = unit_base + i;
            const bool more = i + 1 < u1;
            const Pages<SMALL> next = pages_of(u + 1, more);
            // ---- scores
            f32x4_t s[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[t] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < S::NK; ++c) {
                    const u32x4_t kc = AHEAD ? kr[t][AHEAD ? c : 0] : load_key(u, pages, t, c);
                    if (FMT == CRAFT_KV_BF16) {
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kc), __builtin_bit_cast(bf16x8_t, q[c]), s[t], 0, 0, 0);
                    } else if (FMT == CRAFT_KV_E4M3) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const u32x2_t codes = {kc[2 * e], kc[2 * e + 1]};
                            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(codes), __builtin_bit_cast(bf16x8_t, q[2 * c + e]), s[t], 0, 0, 0);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kc[e]), __uint_as_float(q[c][e]), s[t], 0, 0, 0);
                    }
                }
            }
            float x[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[t][j] = s[t][j] * (FMT == CRAFT_KV_E4M3 ? a.scale_log2 * ks[t][j] : a.scale_log2);
            if (FMT == CRAFT_KV_E4M3) { vs[0] = vs_next[0]; vs[1] = vs_next[1]; }
            // which of the lane's tokens have a page
            bool there[8];
            bool whole = all_seen(u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (SMALL) there[j] = pages.value[j] >= 0;
                else there[j] = pages.tile[j >> 2] >= 0;
                whole = whole && there[j];
            }
            if (SMALL) whole = __all(whole);
            load_keys(u + 1, next);
            // ---- weights
            if (!whole) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int32_t token = u * kUnit + t * 16 + 4 * g + j;
                        if (token < first || token >= len || !there[4 * t + j]) {
                            x[t][j] = -INFINITY;
                            if (FMT == CRAFT_KV_E4M3) vs[t][j] = 0.0f;      // the scale of a row never written
                        }
                    }
            }
            float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
            top = max_of_head(top);
            if (__any(top > z.m)) {
                const float up = fmaxf(z.m, top);
                z.scale(up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(z.m - up));
                z.m = up;
            }
            const float base = z.m == -INFINITY ? 0.0f : z.m;
            float p[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    p[t][j] = __builtin_amdgcn_exp2f(x[t][j] - base);
                    z.l += p[t][j];
                    if (FMT == CRAFT_KV_E4M3) p[t][j] *= vs[t][j];
                }
            // ---- values
            const bool seen = all_seen(u);
            if (FMT == CRAFT_KV_F32) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int c = 0; c < S::NV; ++c) {
                            const typename VWords::type vc = AHEAD ? vr[4 * t + j][AHEAD ? c : 0] : load_value(u, pages, seen, t, j, c);
#pragma unroll
                            for (int e = 0; e < S::CE; ++e)
                                z.acc[c][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word<S::VW>(vc, e)), p[t][j], z.acc[c][e], 0, 0, 0);
                        }
            } else {
                const wide_t pw = {bf16_pair(p[0][0], p[0][1]), bf16_pair(p[0][2], p[0][3]), bf16_pair(p[1][0], p[1][1]), bf16_pair(p[1][2], p[1][3])};
                const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, pw);
#pragma unroll
                for (int c = 0; c < S::NV; ++c) {
                    typename VWords::type vc[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) vc[j] = AHEAD ? vr[j][AHEAD ? c : 0] : load_value(u, pages, seen, j >> 2, j & 3, c);
                    // two neighbouring columns at a time: pairs of tokens out of eight words
#pragma unroll
                    for (int e = 0; e < S::CE / 2; ++e) {
                        uint32_t w[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            w[j] = FMT == CRAFT_KV_BF16 ? word<S::VW>(vc[j], e)
                                   : (e & 1) ? widen_pair<true>(word<S::VW>(vc[j], e >> 1)) : widen_pair<false>(word<S::VW>(vc[j], e >> 1));
                        const wide_t even = {perm(w[1], w[0], 0x05040100u), perm(w[3], w[2], 0x05040100u), perm(w[5], w[4], 0x05040100u), perm(w[7], w[6], 0x05040100u)};
                        const wide_t odd = {perm(w[1], w[0], 0x07060302u), perm(w[3], w[2], 0x07060302u), perm(w[5], w[4], 0x07060302u), perm(w[7], w[6], 0x07060302u)};
                        z.acc[c][2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, even), pf, z.acc[c][2 * e], 0, 0, 0);
                        z.acc[c][2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, odd), pf, z.acc[c][2 * e + 1], 0, 0, 0);
                    }
                }
            }
            load_values(u + 1, next);
            pages = next;
        }

        if (u0 > 0) {
            z.put(s_sums[wave], lane);
            if (lane == 0) s_found[wave] = u1 == n_units ? kEnded : kOpen;
        } else if (u1 == n_units) {
            z.template write<FMT == CRAFT_KV_F32>(a, item_r, head0, n_heads, lane);
        } else {
            open = true;
            open_item = item;
            open_head0 = head0;
            open_heads = n_heads;
            open_end = item_end;
            r = item_r;
        }
    }

    // ---- the waves meet: whoever began an item adds what the following waves found of it
    __syncthreads();
    float *part = a.part + (int64_t)2 * blockIdx.x * State::kFloats;
    if (open) {
        bool ended = false;
        for (int w = wave + 1; w < kWaves && !ended; ++w) {
            z.add(s_sums[w], lane);
            ended = s_found[w] == kEnded;
        }
        if (ended) {
            z.template write<FMT == CRAFT_KV_F32>(a, r, open_head0, open_heads, lane);
        } else {
            z.put(part + State::kFloats, lane);
            if (lane == 0) {
                // joined by the workgroup of the same number in the second launch
                a.desc[4 * blockIdx.x] = r;
                a.desc[4 * blockIdx.x + 1] = open_item;
                a.desc[4 * blockIdx.x + 2] = runs.of(open_end - 1) / kWaves;
            }
        }
    }
    // the item that an earlier workgroup began
    if (wave == 0 && s_found[0] != kNone) {
        z.clear();
        for (int w = 0; w < kWaves; ++w) {
            z.add(s_sums[w], lane);
            if (s_found[w] == kEnded) break;
        }
        z.put(part, lane);
    }
}

// Joins the parts of an item that starts in workgroup blockIdx.x of the first launch and ends in a later one: that
// one's last sums and the first ones of those that follow.
template <int FMT, int DK, int DV>
__global__ __launch_bounds__(kThreads) void join_kernel(AttentionArgs a, int32_t blocks) {
    typedef Shape<FMT, DK, DV> S;
    typedef Sums<S::NV, S::CE> State;
    __shared__ float s_sums[kWaves][State::kFloats];
    const int32_t group = blockIdx.x, r = a.desc[4 * group];
    if (r < 0) return;
    const int32_t item = a.desc[4 * group + 1], last = a.desc[4 * group + 2];
    const int32_t h = item / blocks, block = item - h * blocks;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    State z;
    z.clear();
    for (int32_t w = group + wave; w <= last; w += kWaves) z.add(a.part + (int64_t)(2 * w + (w == group ? 1 : 0)) * State::kFloats, lane);
    if (wave > 0) z.put(s_sums[wave], lane);
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < kWaves && group + w <= last; ++w) z.add(s_sums[w], lane);
    z.template write<FMT == CRAFT_KV_F32>(a, r, h * a.group + block * 16, min(16, a.group - block * 16), lane);
}

template <int FMT, int DK, int DV, bool AHEAD, int WPS>
void launch(const AttentionArgs &a, int32_t blocks, hipStream_t s) {
    const dim3 grid((unsigned)a.workers), block(kThreads);
    if (a.shift < 4) hipLaunchKernelGGL((decode_kernel<FMT, DK, DV, true, AHEAD, WPS>), grid, block, 0, s, a, blocks);
    else hipLaunchKernelGGL((decode_kernel<FMT, DK, DV, false, AHEAD, WPS>), grid, block, 0, s, a, blocks);
    hipLaunchKernelGGL((join_kernel<FMT, DK, DV>), grid, block, 0, s, a, blocks);
}

int padded_dim(const AttentionArgs &a) {
    const int d = std::max(a.dk, a.dv);
    return d <= 64 ? 64 : d <= 128 ? 128 : d <= 256 ? 256 : 576;
}

template <int FMT>
void launch_format(const AttentionArgs &a, int32_t blocks, hipStream_t s) {
    switch (padded_dim(a)) {
    case 64: launch<FMT, 64, 64, true, 2>(a, blocks, s); break;
    case 128: launch<FMT, 128, 128, true, 2>(a, blocks, s); break;
    case 256: launch<FMT, 256, 256, FMT != CRAFT_KV_F32, 2>(a, blocks, s); break;
    default: launch<FMT, 576, 512, false, 1>(a, blocks, s); break;
    }
}

}  // namespace

int32_t attention_workers(const AttentionArgs &a, int32_t num_cu) {
    return (padded_dim(a) == 576 ? 1 : 2) * num_cu;
}

size_t attention_workspace(const AttentionArgs &a, int32_t num_cu) {
    const int dv = padded_dim(a) == 576 ? 512 : padded_dim(a);
    const size_t w = (size_t)attention_workers(a, num_cu);
    return w * 4 * sizeof(int32_t) + w * 2 * (size_t)(16 * dv + 128) * sizeof(float);
}

hipError_t launch_decode_attention(const AttentionArgs &a, hipStream_t s) {
    const int32_t blocks = (a.group + 15) / 16;
    if (a.format == CRAFT_KV_F32) launch_format<CRAFT_KV_F32>(a, blocks, s);
    else if (a.format == CRAFT_KV_BF16) launch_format<CRAFT_KV_BF16>(a, blocks, s);
    else launch_format<CRAFT_KV_E4M3>(a, blocks, s);
    return hipGetLastError();
}

}  // namespace craft
