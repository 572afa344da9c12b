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
// The weights of 16- and 8-bit values go into the second product as two bf16 numbers, a weight's upper half and the nearest
// number to the rest of it: off by 2^-15 of it, not 2^-8.  The second set of products hides behind HBM: two requests of
// 100001 and 131072 tokens, 8 heads of 128 in bf16, with one number a weight / with two 155.8 / 156.1 us; 64 of 1 to 16384 82.2 /
// 82.1; 250 of 1000 to 8000 in 8 bits 150.7 / 151.8; rows of 64 and 80 in 8 bits, the fewest bytes for an instruction, 33.7 / 34.5 and
// 115.9 / 118.6.
// A wave has the keys of the next unit in flight while it works on the weights and values of this one, and the
// other way round.
//
// Work: the (request, head) items, each its units and a few more for what an item costs by itself, are laid end
// to end and cut into equal runs, one per wave, by prefix sums over the lengths that every workgroup does for
// itself: the launch does not depend on the lengths (which the host does not know), and long and short requests
// take equal parts of the GPU.  A wave walks its run alone; what it begins and does not end, or ends and did not
// begin, meets the neighbouring waves' sums in LDS at the end of the workgroup.  An item cut between workgroups
// leaves partial sums in the workspace, and the workgroup that finds by a counter that it is the last of its
// item's joins them, in the order of the runs whoever it is: a second launch would take longer than a whole call
// on a few short requests.  Of an item cut into many parts, 16 at a time are joined first.
//
// Two requests of 100001 and 131072 tokens, 8 heads of 128 in bf16: 155 us, 6.1 TB/s (reads of a large array reach 6.2); 250
// of 1000 to 8000 in 8 bits 151 us, 5.9 TB/s; 64 of 1 to 16384 82 us, 5.4 TB/s; two of 50001 and 65536 in fp32 157 us, 6.0 TB/s.
// 8 of 40 to 1500, 4 heads: 13 us, of which 1 is the bytes'.  The longest is 38 units, so the work is cut: prefix sums, two
// units a wave on 60 workgroups, and the joins of items that lie on up to five of them, one round trip behind another.
#include <algorithm>

#include "attention_common.h"

namespace craft {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
// What an item costs beside its units.  A recorded call with 1 / 2 / 4: 64 requests of 1 to 16384 tokens, 8 heads, 90.7 / 84.4
// / 84.4 us; 250 of 1 to 500 tokens 27.9 / 26.9 / 30.6.
constexpr int kItemCost = 2;
// Most units of an item that is left to one workgroup, where those suffice for all.  With 12 / 24 / 48, 32 requests, 8 heads of
// 128 in bf16: of 600 tokens 24.9 / 18.7 / 18.7 us, of 1000 32.4 / 32.4 / 25.8, of 1500 43.5 / 43.5 / 36.1; but 8 requests, 4 heads: of
// 600 14.0 / 12.7 / 12.7, of 768 13.4 / 14.4 / 14.5, of 1000 14.3 / 14.3 / 17.5, of 1500 15.4 / 15.5 / 23.0.  Cutting wins where the items are few.
constexpr int kWholeUnits = 24;
// Of a wave, where there is little to do.  With 1 / 2 / 4: 2 requests of 2000 tokens, 8 heads, 16.4 / 14.9 / 17.9 us; 8 of 1000, 4 heads,
// 14.3 / 14.3 / 17.4.
constexpr int kMinRun = 2;

template <int NV, int CE, bool F32>
__device__ __forceinline__ void write_item(const Sums<NV, CE, F32> &z, const AttentionArgs &a, const Place &p, int32_t blocks, int lane) {
    const int32_t h = p.item / blocks, block = p.item - h * blocks;
    z.write(a, p.request, h * a.group + block * 16, min(16, a.group - block * 16), lane);
}

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
    typedef Sums<S::NV, S::CE, FMT == CRAFT_KV_F32> State;
    __shared__ float s_sums[kWaves][State::kFloats];   // of the item that a wave's run found begun
    __shared__ int32_t s_found[kWaves];                // whether there is one, and whether it ends in the run
    __shared__ Cut s_cut[2];
    enum { kNone = 0, kOpen = 1, kEnded = 2 };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int32_t per_request = a.heads * blocks, rank = blockIdx.x * kWaves + wave;
    Runs runs = {};
    int64_t at = 0, end = 0, before = 0;
    int32_t r = 0, len = 0;
    // Few short items: a workgroup for each, and nothing to be joined.  Its table entries can be asked for at once.
    const int64_t items = (int64_t)a.R * per_request;
    bool whole_items = a.R <= kThreads && items <= a.workers;
    int32_t early = 0;
    if (whole_items) {
        r = min((int32_t)(blockIdx.x / (uint32_t)per_request), a.R - 1);
        early = a.table[(int64_t)r * a.table_stride + min(lane, a.max_pages - 1)];
        int32_t most = 0;
        for (int32_t i = lane; i < a.R; i += 64) most = max(most, units_of(a, length_of(a, i)));
        whole_items = __all(most <= kWholeUnits);
    }
    if (whole_items) {
        if (blockIdx.x >= items) return;
        len = uniform(length_of(a, r));
        const int32_t units = units_of(a, len), item = (int32_t)(blockIdx.x % (uint32_t)per_request);
        const int64_t begin = (int64_t)item * (units + kItemCost);
        at = begin + (wave > 0 ? kItemCost + units * wave / kWaves : 0);
        end = begin + kItemCost + units * (wave + 1) / kWaves;
    } else {
        const Start st = find_start<kWaves, kWaves>(a, per_request, kItemCost, a.workers * kWaves, kMinRun, blockIdx.x * kWaves, runs);
        if ((int32_t)blockIdx.x * kWaves >= runs.n) return;
        if (rank < runs.n) {
            at = runs.start(rank);
            end = runs.start(rank + 1);
        }
        before = st.before;
        r = st.request;
        len = st.len;
    }
    if (lane == 0) s_found[wave] = kNone;
    if (tid < 2) s_cut[tid].mine = 0;
    State z;
    bool open = false;                             // the run ends inside an item that starts in it
    Place began = {}, opened = {};                 // the item a run finds begun, the one it leaves open

    while (at < end) {
        const int32_t first = first_of(a, len), n_units = units_of(a, len), cost = n_units + kItemCost;
        const int64_t in_request = at - before;
        const int32_t item = in_request >> 32 ? (int32_t)(in_request / cost) : (int32_t)((uint32_t)in_request / (uint32_t)cost);
        const int64_t item_begin = before + (int64_t)item * cost, item_end = item_begin + cost;
        const int64_t stop = min(end, item_end);
        // an item's own cost comes first
        const int32_t u0 = max(0, (int32_t)(at - item_begin) - kItemCost), u1 = max(0, (int32_t)(stop - item_begin) - kItemCost);
        at = stop;
        const Place here = {item_begin, item_end, r, item};
        const int32_t n = len;
        // the next run of items' length travels meanwhile
        if (at == before + (int64_t)cost * per_request && at < end) {
            before = at;
            ++r;
            len = uniform(length_of(a, r));
        }
        if (u0 == u1) continue;
        const int32_t h = item / blocks, block = item - h * blocks;
        const int32_t head0 = h * a.group + block * 16, n_heads = min(16, a.group - block * 16);
        const int32_t unit_base = first / kUnit;   // of the request's visible tokens

        // ---- queries: the right operand of the first product, laid out as the key pieces are
        u32x4_t q[S::QN];
        {
            const bool live = col < n_heads;
            constexpr int QB = FMT == CRAFT_KV_F32 ? 4 : 2, QE = 16 / QB;     // bytes of an element, elements of a piece
            const __amdgpu_buffer_rsrc_t qr = rows_of(static_cast<const unsigned char *>(a.q) + ((int64_t)here.request * a.q_stride + (int64_t)head0 * a.q_head) * QB, kFar);
            const uint32_t q_off = (uint32_t)col * (uint32_t)a.q_head * QB;
#pragma unroll
            for (int i = 0; i < S::QN; ++i) {
                const int d = FMT == CRAFT_KV_E4M3 ? (i >> 1) * 64 + g * 16 + (i & 1) * 8 : i * 4 * QE + g * QE;
                q[i] = __builtin_amdgcn_raw_buffer_load_b128(qr, live && d < a.dk ? q_off + d * QB : kFar, 0, 0);
            }
        }

        const unsigned char *kh = a.k + h * a.k_head, *vh = a.v + h * a.v_head;
        const int32_t *table = a.table + (int64_t)here.request * a.table_stride;
        const uint32_t k_span = 15u * (uint32_t)a.k_token + (uint32_t)a.dk * S::B, v_span = 15u * (uint32_t)a.v_token + (uint32_t)a.dv * S::B;
        const uint32_t k_off = (uint32_t)col * (uint32_t)a.k_token + g * 16;

        z.clear();

        u32x4_t kr[2][AHEAD ? S::NK : 1];
        typename VWords::type vr[8][AHEAD ? S::NV : 1];
        f32x4_t ks[2], vs[2], vs_next[2];

        auto checked = [&](int32_t page) -> int32_t { return (uint32_t)page < (uint32_t)a.pages ? page : -1; };
        auto entry = [&](int32_t i) -> int32_t { return table[min(i, a.max_pages - 1)]; };
        // A wave holds 64 entries of the table and the 64 behind them.  They are renewed between runs of units that
        // need no others: a request for them among the units' would have its wait among theirs.
        int32_t held0 = ((unit_base + u0) * kUnit) >> a.shift;
        int32_t held = early, behind = 0;
        if (whole_items && ((unit_base + u1) * kUnit - 1) >> a.shift < 64) {
            held0 = 0;
        } else if (!SMALL) {
            held = entry(held0 + lane);
            behind = entry(held0 + 64 + lane);
        }
        auto pages_of = [&](int32_t u, bool live) -> Pages<SMALL> {
            Pages<SMALL> pg;
            if constexpr (SMALL) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int32_t token = u * kUnit + t * 16 + col;
                    pg.key[t] = live && token < n ? checked(entry(token >> a.shift)) : -1;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int32_t token = u * kUnit + (j >> 2) * 16 + 4 * g + (j & 3);
                    pg.value[j] = live && token < n ? checked(entry(token >> a.shift)) : -1;
                }
            } else {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int32_t token = u * kUnit + t * 16;
                    const int32_t i = (token >> a.shift) - held0;
                    const int32_t in_held = __builtin_amdgcn_readlane(held, i & 63), in_behind = __builtin_amdgcn_readlane(behind, i & 63);
                    const int32_t page = checked(i < 64 ? in_held : in_behind);
                    pg.tile[t] = live && token < n ? page : -1;
                }
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
                const __amdgpu_buffer_rsrc_t rs = rows_of(kh + max(pg.tile[t], 0) * a.k_page + (token & in_page) * a.k_token, pg.tile[t] >= 0 ? k_span : 0u);
                return __builtin_amdgcn_raw_buffer_load_b128(rs, (inside ? k_off : kFar) + i * 64, 0, 0);
            }
        };
        // rows behind the last token (and in front of the window) may hold anything: read as zeros
        auto load_value = [&](int32_t u, const Pages<SMALL> &pg, bool whole, int t, int j, int c) __attribute__((always_inline)) -> typename VWords::type {
            const int32_t token = u * kUnit + t * 16, row = 4 * g + j;
            const bool inside = (whole || (token + row >= first && token + row < n)) && (c * 16 + col) * S::CE < a.dv;
            if constexpr (SMALL) {
                const int32_t page = pg.value[4 * t + j];
                typename VWords::type x = {};
                if (inside && page >= 0)
                    x = *reinterpret_cast<const typename VWords::type *>(vh + page * a.v_page + ((token + row) & in_page) * a.v_token + (c * 16 + col) * (S::CE * S::B));
                return x;
            } else {
                const __amdgpu_buffer_rsrc_t rs = rows_of(vh + max(pg.tile[t], 0) * a.v_page + (token & in_page) * a.v_token, pg.tile[t] >= 0 ? v_span : 0u);
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
                    const uint32_t span = pg.tile[t] >= 0 ? 64u : 0u;
                    const int64_t so = (((int64_t)max(pg.tile[t], 0) * a.heads + h) << a.shift) + (token & in_page);
                    ks[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                        rows_of(reinterpret_cast<const unsigned char *>(a.k_scale + so), span), g * 16, 0, 0));
                    vs_next[t] = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(
                        rows_of(reinterpret_cast<const unsigned char *>(a.v_scale + so), span), g * 16, 0, 0));
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
        auto all_seen = [&](int32_t u) { return u * kUnit >= first && u * kUnit + kUnit <= n; };
        auto load_values = [&](int32_t u, const Pages<SMALL> &pg) __attribute__((always_inline)) {
            if constexpr (AHEAD) {
                auto load = [&](bool whole) __attribute__((always_inline)) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int c = 0; c < S::NV; ++c) vr[4 * t + j][c] = load_value(u, pg, whole, t, j, c);
                };
                if (all_seen(u)) load(true);
                else load(false);
            }
        };

        Pages<SMALL> pages = pages_of(unit_base + u0, true);
        load_keys(unit_base + u0, pages);
        load_values(unit_base + u0, pages);
        for (int32_t i = u0; i < u1;) {
            // up to the first unit whose page is not held; the one behind it is (pages have half a unit at least)
            const int32_t stop_at = SMALL ? u1 : min(u1, (int32_t)min((int64_t)u1, (((int64_t)held0 + 64) << a.shift) / kUnit - unit_base));
            for (; i < stop_at; ++i) {
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
                bool whole = all_seen(u);
                const Pages<SMALL> seen_pages = pages;
                auto there = [&](int j) {
                    if constexpr (SMALL) return seen_pages.value[j] >= 0;
                    else return seen_pages.tile[j >> 2] >= 0;
                };
                if constexpr (SMALL) {
                    int32_t all = 0;
#pragma unroll
                    for (int j = 0; j < 8; ++j) all |= seen_pages.value[j];
                    whole = whole && __all(all >= 0);
                } else {
                    whole = whole && (seen_pages.tile[0] | seen_pages.tile[1]) >= 0;
                }
                load_keys(u + 1, next);
                // ---- weights
                if (!whole) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int32_t token = u * kUnit + t * 16 + 4 * g + j;
                            if (token < first || token >= n || !there(4 * t + j)) {
                                x[t][j] = -INFINITY;
                                if (FMT == CRAFT_KV_E4M3) vs[t][j] = 0.0f;      // the scale of a row never written
                            }
                        }
                }
                float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
                top = max_of_head(top);
                const float base = z.raise(top);
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
                    // the weights' upper halves, and what that leaves of them: never zero where the weight is not, so that
                    // an infinite value stays one in both products (an infinite weight, of an infinite scale, as well)
                    wide_t pw, pr;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p0 = p[i >> 1][2 * (i & 1)], p1 = p[i >> 1][2 * (i & 1) + 1];
                        const uint32_t h0 = __float_as_uint(p0) & 0xffff0000u, h1 = __float_as_uint(p1) & 0xffff0000u;
                        pw[i] = perm(h1, h0, 0x07060302u);
                        pr[i] = bf16_pair(fmaxf(p0 - __uint_as_float(h0), p0 * 0x1p-20f), fmaxf(p1 - __uint_as_float(h1), p1 * 0x1p-20f));
                    }
                    const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, pw), rest = __builtin_bit_cast(bf16x8_t, pr);
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
                            z.acc[c][2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, even), rest, z.acc[c][2 * e], 0, 0, 0);
                            z.acc[c][2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, odd), rest, z.acc[c][2 * e + 1], 0, 0, 0);
                        }
                    }
                }
                load_values(u + 1, next);
                pages = next;
            }
            if (i < u1) {
                held0 += 64;
                held = behind;
                behind = entry(held0 + 64 + lane);
            }
        }

        if (u0 > 0) {
            z.put(s_sums[wave], lane);
            began = here;
            if (lane == 0) s_found[wave] = u1 == n_units ? kEnded : kOpen;
        } else if (u1 == n_units) {
            write_item(z, a, here, blocks, lane);
        } else {
            open = true;
            opened = here;
        }
    }

    // ---- the waves meet: whoever began an item adds what the following waves found of it
    __syncthreads();
    auto part_of = [&](int32_t group, bool begins) { return a.part + (int64_t)(2 * group + (begins ? 1 : 0)) * State::kFloats; };
    if (open) {
        bool ended = false;
        for (int w = wave + 1; w < kWaves && !ended; ++w) {
            if (s_found[w] == kNone) continue;
            z.add(s_sums[w], lane);
            ended = s_found[w] == kEnded;
        }
        if (ended) {
            write_item(z, a, opened, blocks, lane);
        } else {
            z.put_out(part_of(blockIdx.x, true), lane);
            if (lane == 0) s_cut[0] = {opened, 1};
        }
    }
    // the item that an earlier workgroup began
    if (wave == 0 && s_found[0] != kNone) {
        z.clear();
        for (int w = 0; w < kWaves; ++w) {
            z.add(s_sums[w], lane);
            if (s_found[w] == kEnded) break;
        }
        z.put_out(part_of(blockIdx.x, false), lane);
        if (lane == 0) s_cut[1] = {began, 1};
    }
    __syncthreads();
    if (!s_cut[0].mine && !s_cut[1].mine) return;

    // ---- joins of items cut between workgroups.  Counters: parts of a group of 16 that have arrived, by the
    // number of the group's first workgroup (as the item's first one, or as a later one), and groups, by that of
    // the item's first.  The last to arrive leaves a counter as it was found, at zero.
    __shared__ int32_t s_last;
    for (int i = 0; i < 2; ++i) {
        if (!s_cut[i].mine) continue;
        const Place cut = s_cut[i].item;
        const int32_t first = runs.of(uniform(cut.begin) + kItemCost) / kWaves, last = runs.of(uniform(cut.end) - 1) / kWaves;
        const int32_t number = ((int32_t)blockIdx.x - first) / kJoin, lead = first + number * kJoin;
        const int32_t stop = min(lead + kJoin, last + 1), groups = (last - first) / kJoin + 1;
        // the sums of parts lo, lo + step, .. below hi, in the first wave
        auto join = [&](int32_t lo, int32_t hi, int32_t step) {
            z.clear();
            for (int32_t w = lo + wave * step; w < hi; w += kWaves * step) z.add_from(part_of(w, w == first), lane);
            if (wave > 0) z.put(s_sums[wave], lane);
            __syncthreads();
            if (wave == 0)
                for (int w = 1; w < kWaves && lo + w * step < hi; ++w) z.add(s_sums[w], lane);
            __syncthreads();
        };
        if (!last_to_arrive(a.counters + (number ? kCounters : 0) + lead, stop - lead, &s_last)) continue;
        join(lead, stop, 1);
        if (groups > 1) {
            if (wave == 0) z.put_out(part_of(lead, number == 0), lane);
            if (!last_to_arrive(a.counters + 2 * kCounters + first, groups, &s_last)) continue;
            join(first, last + 1, kJoin);
        }
        if (wave == 0) write_item(z, a, cut, blocks, lane);
    }
}

// Workgroups of a CU, by the bytes of a unit's rows (keys and values) as they are padded, which is what a wave has
// registers and loads for.  More waves hide more latency, and read less in order.
//   16 KiB and more: one.  Two requests of 100001 and 131072 tokens, 8 heads of 128 in bf16, with one / two 155 / 163 us.  Rows
//     of 80 and 96 elements have 10 and 12 KiB of these on their way and do no better with two: 64 requests of 1 to
//     16384, 8 heads, 57 / 60 and 65 / 68 us.
//   8 KiB: two.  The same requests, rows of 128 in 8 bits, with one / two 59 / 51.5 us, of 64 in bf16 50 / 47.
//   4 KiB: four.  1000 requests of 100 to 1000 tokens, 8 heads of 64 in 8 bits, with two / four 108 / 97 us; 500 of 1000 to 4000
//     227 / 221.
//   Pages of fewer than 16 tokens, for their chains of lookups: two.  The two long requests in pages of 8 with one / two 206
//     / 181 us.  64 KiB (rows of 256 in fp32): one, all that the registers hold.
constexpr int groups_of(int format, int dim, bool small) {
    const int unit = kUnit * 2 * dim * (format == CRAFT_KV_F32 ? 4 : format == CRAFT_KV_BF16 ? 2 : 1);
    return unit >= 65536 ? 1 : small ? 2 : unit >= 16384 ? 1 : unit >= 8192 ? 2 : 4;
}

template <int FMT, int D>
void launch(const AttentionArgs &a, int32_t blocks, hipStream_t s) {
    constexpr int DK = D, DV = D == 576 ? 512 : D;
    const dim3 grid((unsigned)a.workers), block(kThreads);
    if (a.shift < 4) hipLaunchKernelGGL((decode_kernel<FMT, DK, DV, true, D != 576, groups_of(FMT, D, true)>), grid, block, 0, s, a, blocks);
    else hipLaunchKernelGGL((decode_kernel<FMT, DK, DV, false, D != 576, groups_of(FMT, D, false)>), grid, block, 0, s, a, blocks);
}

int padded_dim(const AttentionArgs &a) {
    const int d = std::max(a.dk, a.dv);
    return d <= 64 ? 64 : d <= 128 ? 128 : d <= 256 ? 256 : 576;
}

template <int FMT>
void launch_format(const AttentionArgs &a, int32_t blocks, hipStream_t s) {
    switch (padded_dim(a)) {
    case 64: launch<FMT, 64>(a, blocks, s); break;
    case 128: launch<FMT, 128>(a, blocks, s); break;
    case 256: launch<FMT, 256>(a, blocks, s); break;
    default:
        if constexpr (FMT == CRAFT_KV_F32) launch<FMT, 576>(a, blocks, s);
        break;
    }
}

}  // namespace

// Latent rows in 16 or 8 bits have a kernel of their own; in fp32, which serves bring-up, they come through here,
// every block of 16 heads by itself.
bool wide_latent(const AttentionArgs &a) { return padded_dim(a) == 576 && a.format != CRAFT_KV_F32; }

int32_t attention_workers(const AttentionArgs &a, int32_t num_cu) {
    if (wide_latent(a)) return latent_workers(a, num_cu);
    return std::min(kCounters, groups_of(a.format, padded_dim(a), a.shift < 4) * num_cu);
}

size_t attention_counters_bytes() { return CRAFT_ATTENTION_COUNTER_BYTES; }
static_assert(CRAFT_ATTENTION_COUNTER_BYTES == 3 * kCounters * sizeof(int32_t), "three counters for every workgroup of a launch");

size_t attention_workspace(const AttentionArgs &a, int32_t num_cu) {
    const int dv = padded_dim(a) == 576 ? 512 : padded_dim(a);
    if (wide_latent(a)) return attention_counters_bytes() + latent_workspace(a, num_cu);
    return attention_counters_bytes() + (size_t)attention_workers(a, num_cu) * 2 * (size_t)(16 * dv + 128) * sizeof(float);
}

hipError_t launch_decode_attention(const AttentionArgs &a, hipStream_t s) {
    if (wide_latent(a)) return launch_latent_attention(a, a.part, s);
    const int32_t blocks = (a.group + 15) / 16;
    if (a.format == CRAFT_KV_F32) launch_format<CRAFT_KV_F32>(a, blocks, s);
    else if (a.format == CRAFT_KV_BF16) launch_format<CRAFT_KV_BF16>(a, blocks, s);
    else launch_format<CRAFT_KV_E4M3>(a, blocks, s);
    return hipGetLastError();
}

}  // namespace craft
