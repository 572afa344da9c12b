// Paged key/value cache: block tables and slot maps of a serving step, and the writes of new rows.
//
// Tables.  With n the tokens a request has, a the ones it gets and P the tokens of a page, it takes
// need = ceil((n + a) / P) - ceil(n / P) pages.  Three prefix sums over the requests (tokens, pages taken,
// pages given back) decide who is served and give every token and page its place: one workgroup does them.
// What follows is independent per token: its page comes out of the table or, for a new page, out of the ring of
// free pages, and the token that is first on its page writes the table entry.  The bytes are next to nothing; a
// step is a chain of a few dependent round trips (lengths, ring, slots).  So a small step is one launch, and where
// no request gets more than one token, as in decoding, its thread writes it; otherwise a token's request is found
// by binary search among the token offsets in LDS.  A large step fills in a second launch on many CUs.
//
// Writes.  Bound by HBM: every row read once and written once, 16 bytes per lane.  In 8 bits the lanes of a
// row share its maximum (codes and scales as of expert weights).
#include <algorithm>

#include "e4m3.h"
#include "kernels.h"
#include "shares.h"

namespace craft {
namespace {

// ------------------------------------------------------------------------ tables

constexpr int kScanThreads = 1024;                // also the most requests of a step of one launch: one per thread
constexpr int kFillThreads = 256;
// Tokens a thread fills in.  A recorded step with 1 / 2 / 8: 1500 requests of up to 1024 tokens, 211313 in all, 10.7 / 10.1 / 16.8 us;
// 1000 requests with 5974 tokens 7.2 / 8.3 / 14.7.
constexpr int kFillTokens = 2;
// Most requests of which a filling workgroup keeps its own copy (48 KiB of LDS), for its searches.  With the copy / without, 1500
// requests and 211313 tokens 10.1 / 11.3 us, 4000 of one token each 17.9 / 18.7.
constexpr int kFillRequests = 4096;

// Sums over some requests, in 32 bits that saturate: what exceeds 2^31 exceeds every bound there is.
struct Counts {
    uint32_t tokens, need, back;
};
__device__ __forceinline__ Counts operator+(const Counts &a, const Counts &b) {
    return {__builtin_elementwise_add_sat(a.tokens, b.tokens), __builtin_elementwise_add_sat(a.need, b.need),
            __builtin_elementwise_add_sat(a.back, b.back)};
}
// x of the lane DPP names, 0 where there is none
template <int DPP, int ROWS> __device__ __forceinline__ uint32_t lane_of(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, DPP, ROWS, 0xf, false);
}
template <int DPP, int ROWS> __device__ __forceinline__ Counts lane_of(const Counts &x) {
    return {lane_of<DPP, ROWS>(x.tokens), lane_of<DPP, ROWS>(x.need), lane_of<DPP, ROWS>(x.back)};
}
// Sums over a wave's lanes up to each: within rows of 16 lanes (shifts by 1, 2, 4, 8), then the last lane of a row
// to the next one, and of the second row to the upper half.
__device__ __forceinline__ Counts wave_sums(Counts x) {
    x = x + lane_of<0x111, 0xf>(x);
    x = x + lane_of<0x112, 0xf>(x);
    x = x + lane_of<0x114, 0xf>(x);
    x = x + lane_of<0x118, 0xf>(x);
    x = x + lane_of<0x142, 0xa>(x);
    x = x + lane_of<0x143, 0xc>(x);
    return x;
}
// i mod n for i of either sign
__device__ __forceinline__ uint32_t ring_place(int64_t i, int64_t n) {
    if ((uint64_t)i >> 32 == 0) return (uint32_t)i % (uint32_t)n;
    const int64_t m = i % n;
    return (uint32_t)(m < 0 ? m + n : m);
}

struct Request {
    int32_t n, asked, have, need, back;
};
__device__ __forceinline__ Request request_of(const KvTablesArgs &a, int32_t add, int32_t len) {
    const int64_t cap = (int64_t)a.max_pages << a.shift;
    Request q;
    q.n = (int32_t)min((int64_t)max(len, 0), cap);
    q.asked = add > 0 && (int64_t)q.n + add <= cap ? add : 0;
    const int64_t up = (1ll << a.shift) - 1;
    q.have = (int32_t)((q.n + up) >> a.shift);
    q.need = (int32_t)(((int64_t)q.n + q.asked + up) >> a.shift) - q.have;
    q.back = add < 0 ? q.have : 0;
    return q;
}

// One token: its page, the table entry if the page starts with it, its slot.
__device__ __forceinline__ void put_token(const KvTablesArgs &a, int32_t t, int32_t r, int32_t first, int32_t n,
                                          int32_t page_off, uint32_t head) {
    const int32_t pos = n + (t - first);
    const int32_t pidx = pos >> a.shift, within = pos & ((1 << a.shift) - 1);
    const int32_t have = (int32_t)(((int64_t)n + (1ll << a.shift) - 1) >> a.shift);
    int32_t *entry = a.table + (int64_t)r * a.table_stride + pidx;
    int32_t page;
    if (pidx >= have) {
        uint32_t i = head + (uint32_t)page_off + (uint32_t)(pidx - have);       // below 2 pages, < 2^32
        if (i >= (uint32_t)a.pages) i -= (uint32_t)a.pages;
        page = a.ring[i];
        if (within == 0) *entry = page;
    } else {
        page = *entry;
    }
    a.slots[t] = (uint32_t)page < (uint32_t)a.pages ? (page << a.shift) + within : -1;
    if (a.positions) a.positions[t] = pos;
}

// The pages of the ended requests among the 64 from r0 on, one request after the other by a whole wave.
// n, back_off: of request r0 + lane; tail: the first place behind the free pages.
__device__ __forceinline__ void give_back(const KvTablesArgs &a, int32_t r0, bool ended, int32_t n, uint32_t back_off, uint32_t tail) {
    const int lane = threadIdx.x & 63;
    unsigned long long m = __ballot(ended && n > 0);
    while (m) {
        const int j = __ffsll((long long)m) - 1;
        m &= m - 1;
        const int32_t have = (int32_t)(((int64_t)__shfl(n, j, 64) + (1ll << a.shift) - 1) >> a.shift);
        const uint32_t base = (uint32_t)(((uint64_t)tail + (uint32_t)__shfl((int)back_off, j, 64)) % (uint64_t)a.pages);
        const int32_t *row = a.table + (int64_t)(r0 + j) * a.table_stride;
        for (int32_t c = lane; c < have; c += 64) a.ring[(base + (uint32_t)c) % (uint32_t)a.pages] = row[c];
    }
}
__device__ __forceinline__ void no_token(const KvTablesArgs &a, int64_t t) {
    a.slots[t] = -1;
    if (a.positions) a.positions[t] = -1;
}

// FUSED: the whole step in this launch, of THREADS requests at most.  Otherwise the workspace gets what the filling
// launch needs: the ring's first free entry and its end, the number of tokens, then lengths, page and back offsets.
template <bool FUSED, int THREADS>
__global__ __launch_bounds__(THREADS) void tables_scan_kernel(KvTablesArgs a) {
    constexpr int kWaves = THREADS / 64;
    __shared__ Counts wave_sum[kWaves];
    __shared__ uint32_t wave_most[kWaves][2], wave_asked[kWaves];
    __shared__ int32_t s_off[FUSED ? THREADS : 1], s_n[FUSED ? THREADS : 1], s_page[FUSED ? THREADS : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t taken = a.pool[0], returned = a.pool[1];
    // this thread's requests: a run of `per`
    const int32_t per = FUSED ? 1 : share_of<THREADS>(a.R);
    const int64_t r0 = (int64_t)tid * per, r1 = min((int64_t)a.R, r0 + per);
    Counts sum = {0, 0, 0};
    Request q = {0, 0, 0, 0, 0};
    int32_t add = 0;
    for (int64_t r = r0; r < r1; ++r) {
        add = a.add[r];
        q = request_of(a, add, a.lens[r]);
        sum = sum + Counts{(uint32_t)q.asked, (uint32_t)q.need, (uint32_t)q.back};
    }
    const Counts incl = wave_sums(sum);
    if (lane == 63) wave_sum[wave] = incl;
    const bool several = __any(q.asked > 1);       // one launch: some request gets more than one token
    if (FUSED && lane == 0) wave_asked[wave] = several;
    const uint32_t spare = (uint32_t)min(max(returned - taken, (int64_t)0), a.pages);
    const uint32_t head = ring_place(taken, a.pages), tail = ring_place(returned, a.pages);
    __syncthreads();
    Counts before = {0, 0, 0}, total = {0, 0, 0};
    bool search = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w == wave) before = total;
        total = total + wave_sum[w];
        if (FUSED) search = search || wave_asked[w];
    }
    // the sums in front of this thread's requests: of the waves before, and of the lanes before
    before = before + lane_of<0x138, 0xf>(incl);
    uint32_t tokens = total.tokens, pages = total.need;
    if (total.need > spare || total.tokens > (uint32_t)a.max_new) {
        // Not all are served.  Sums only grow, so those that ask for anything and are served are the first few.
        tokens = pages = 0;
        Counts b = before;
        for (int64_t r = r0; r < r1; ++r) {
            const Request p = FUSED ? q : request_of(a, a.add[r], a.lens[r]);
            b = b + Counts{(uint32_t)p.asked, (uint32_t)p.need, (uint32_t)p.back};
            if (b.need <= spare && b.tokens <= (uint32_t)a.max_new) {
                tokens = b.tokens;
                pages = b.need;
            }
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            tokens = max(tokens, (uint32_t)__shfl_xor((int)tokens, d, 64));
            pages = max(pages, (uint32_t)__shfl_xor((int)pages, d, 64));
        }
        if (lane == 0) { wave_most[wave][0] = tokens; wave_most[wave][1] = pages; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            tokens = max(tokens, wave_most[w][0]);
            pages = max(pages, wave_most[w][1]);
        }
    }
    const uint32_t back_off = before.back;
    for (int64_t r = r0; r < r1; ++r) {
        const int32_t ad = FUSED ? add : a.add[r];
        const Request p = FUSED ? q : request_of(a, ad, a.lens[r]);
        const Counts here = {(uint32_t)p.asked, (uint32_t)p.need, (uint32_t)p.back}, after = before + here;
        const int32_t off = (int32_t)min(before.tokens, tokens), page_off = (int32_t)min(before.need, pages);
        const bool served = after.need <= spare && after.tokens <= (uint32_t)a.max_new;
        a.token_off[r] = off;
        // lens_out may be lens: this thread has read its requests, and nobody else reads them
        a.lens_out[r] = ad < 0 ? 0 : p.n + (served ? p.asked : 0);
        if (!FUSED) {
            a.ws_len[r] = p.n;
            a.ws_page[r] = page_off;
            a.ws_back[r] = (int32_t)before.back;
        } else if (!search) {
            if (served && p.asked) put_token(a, off, (int32_t)r, off, p.n, page_off, head);
        } else {
            s_off[r] = off;
            s_n[r] = p.n;
            s_page[r] = page_off;
        }
        before = after;
    }
    if (tid == 0) {
        a.token_off[a.R] = (int32_t)tokens;
        // every thread has read the counters before the barrier above
        a.pool_out[0] = taken + pages;
        a.pool_out[1] = returned + total.back;
        if (!FUSED) {
            a.ws_ctrl[0] = (int32_t)head;
            a.ws_ctrl[1] = (int32_t)tail;
            a.ws_ctrl[2] = (int32_t)tokens;
        }
    }
    if (FUSED) {
        if (search) {
            __syncthreads();
            for (int32_t t = tid; t < (int32_t)tokens; t += THREADS) {
                int32_t lo = 0, hi = a.R;          // the last request that starts at t or before
                while (hi - lo > 1) {
                    const int32_t mid = (lo + hi) >> 1;
                    if (s_off[mid] <= t) lo = mid; else hi = mid;
                }
                put_token(a, t, lo, s_off[lo], s_n[lo], s_page[lo], head);
            }
        }
        for (int64_t t = (int64_t)tokens + tid; t < a.max_new; t += THREADS) no_token(a, t);
        give_back(a, wave * 64, tid < a.R && add < 0, q.n, back_off, tail);
    }
}

// Workgroups below `token_groups` take kFillTokens tokens a thread; the others give back the pages of 256
// requests each.  IN_LDS: what the tokens need of the requests fits there.
template <bool IN_LDS>
__global__ __launch_bounds__(kFillThreads) void tables_fill_kernel(KvTablesArgs a, int32_t token_groups) {
    constexpr int kRoom = IN_LDS ? kFillRequests : 1;
    __shared__ int32_t s_off[kRoom], s_n[kRoom], s_page[kRoom];
    if ((int32_t)blockIdx.x >= token_groups) {
        const int64_t r = (int64_t)(blockIdx.x - token_groups) * kFillThreads + threadIdx.x;
        const bool live = r < a.R;
        const int32_t add = live ? a.add[r] : 0, n = live ? a.ws_len[r] : 0, back = live ? a.ws_back[r] : 0;
        give_back(a, (int32_t)(r - (threadIdx.x & 63)), add < 0, n, (uint32_t)back, (uint32_t)a.ws_ctrl[1]);
        return;
    }
    if (IN_LDS) {
        for (int32_t i = threadIdx.x; i < a.R; i += kFillThreads) {
            s_off[i] = a.token_off[i];
            s_n[i] = a.ws_len[i];
            s_page[i] = a.ws_page[i];
        }
    }
    const int32_t tokens = a.ws_ctrl[2];
    const uint32_t head = (uint32_t)a.ws_ctrl[0];
    if (IN_LDS) __syncthreads();
    const int64_t t0 = (int64_t)blockIdx.x * (kFillThreads * kFillTokens) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kFillTokens; ++i) {
        const int64_t t = t0 + i * kFillThreads;
        if (t >= a.max_new) break;
        if (t < tokens) {
            int32_t lo = 0, hi = a.R;
            while (hi - lo > 1) {
                const int32_t mid = lo + ((hi - lo) >> 1);
                if ((IN_LDS ? s_off[mid] : a.token_off[mid]) <= t) lo = mid; else hi = mid;
            }
            if (IN_LDS) put_token(a, (int32_t)t, lo, s_off[lo], s_n[lo], s_page[lo], head);
            else put_token(a, (int32_t)t, lo, a.token_off[lo], a.ws_len[lo], a.ws_page[lo], head);
        } else {
            no_token(a, t);
        }
    }
}

// ------------------------------------------------------------------------ writes

// Rows of a token: its key rows, then its value rows.  A thread copies one 16-byte piece.
__global__ __launch_bounds__(256) void append_copy_kernel(KvAppendArgs a, uint32_t k_pieces, uint32_t pieces, uint32_t first) {
    const int64_t i = ((int64_t)first + blockIdx.x) * 256 + threadIdx.x;
    if (i >= a.T * pieces) return;
    const int64_t t = a.T * pieces <= 0xffffffffll ? (int64_t)((uint32_t)i / pieces) : i / pieces;
    uint32_t c = (uint32_t)(i - t * pieces);
    const bool is_v = c >= k_pieces;
    if (is_v) c -= k_pieces;
    const int32_t slot = a.slots[t];
    const uint32_t row = (uint32_t)(is_v ? a.v_row : a.k_row);      // pieces of a row
    const uint32_t h = c / row, within = c - h * row;
    const u32x4_t x = *reinterpret_cast<const u32x4_t *>((is_v ? a.v : a.k) + t * (is_v ? a.v_stride : a.k_stride) + (int64_t)c * 16);
    if ((uint32_t)slot >= (uint32_t)a.slots_total) return;
    const int64_t page = slot >> a.shift, place = slot & ((1 << a.shift) - 1);
    unsigned char *to = is_v ? a.cv + page * a.cv_page + h * a.cv_head + place * a.cv_token
                             : a.ck + page * a.ck_page + h * a.ck_head + place * a.ck_token;
    *reinterpret_cast<u32x4_t *>(to + within * 16) = x;
}

// LANES lanes per row (the least power of two that holds the longer kind's pieces of 8 elements, 64 at most),
// ITER pieces per lane.
template <int LANES, int ITER>
__global__ __launch_bounds__(256) void append_e4m3_kernel(KvAppendArgs a, uint32_t rows, uint32_t first) {
    const int64_t i = (((int64_t)first + blockIdx.x) * 256 + threadIdx.x) / LANES;
    const int lane = threadIdx.x & (LANES - 1);
    const bool live = i < a.T * rows;
    const int64_t t = live ? (a.T * rows <= 0xffffffffll ? (int64_t)((uint32_t)i / rows) : i / rows) : 0;
    const uint32_t hv = live ? (uint32_t)(i - t * rows) : 0u;
    const bool is_v = hv >= (uint32_t)a.heads;
    const uint32_t h = is_v ? hv - a.heads : hv;
    const int32_t slot = live ? a.slots[t] : -1;
    const int32_t pieces = is_v ? a.v_row : a.k_row;
    const unsigned char *src = (is_v ? a.v : a.k) + t * (is_v ? a.v_stride : a.k_stride) + (int64_t)h * pieces * 16;
    const u32x4_t none = {0u, 0u, 0u, 0u};
    u32x4_t x[ITER];
    float amax = 0.0f;
#pragma unroll
    for (int j = 0; j < ITER; ++j) {
        const int c = j * LANES + lane;
        x[j] = live && c < pieces ? *reinterpret_cast<const u32x4_t *>(src + c * 16) : none;
        amax = max_abs(amax, x[j]);
    }
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d, 64));
    if ((uint32_t)slot >= (uint32_t)a.slots_total) return;
    const RowScale rs = row_scale(amax);
    const int64_t page = slot >> a.shift, place = slot & ((1 << a.shift) - 1);
    unsigned char *to = is_v ? a.cv + page * a.cv_page + h * a.cv_head + place * a.cv_token
                             : a.ck + page * a.ck_page + h * a.ck_head + place * a.ck_token;
#pragma unroll
    for (int j = 0; j < ITER; ++j) {
        const int c = j * LANES + lane;
        if (c < pieces) *reinterpret_cast<u32x2_t *>(to + c * 8) = eight_codes(x[j], rs);
    }
    if (lane == 0) (is_v ? a.v_scale : a.k_scale)[((page * a.heads + h) << a.shift) + place] = rs.s;
}

template <int LANES, int ITER>
void launch_e4m3(const KvAppendArgs &a, hipStream_t s) {
    const uint32_t rows = (uint32_t)a.heads * (a.v ? 2u : 1u);
    const int64_t groups = (a.T * rows * LANES + 255) / 256;
    constexpr int64_t kMost = (1ll << 31) / 256;   // a launch has fewer than 2^32 threads
    for (int64_t g = 0; g < groups; g += kMost)
        hipLaunchKernelGGL((append_e4m3_kernel<LANES, ITER>), dim3((unsigned)std::min(kMost, groups - g)), dim3(256), 0, s, a, rows, (uint32_t)g);
}

}  // namespace

// A step of one launch is one workgroup's: from about kFusedTokens tokens on many CUs do the filling sooner than one does,
// in spite of the second launch.  One launch / two, recorded: 1695 tokens of 1000 requests 7.2 / 8.3 us, 3086 tokens 8.4 / 8.3
// (called one by one 8.6 / 9.3), 5974 tokens 11.4 / 8.3; 4640 tokens of 200 requests 19.3 / 6.6.
constexpr int32_t kFusedTokens = 4096;

hipError_t launch_kv_tables(const KvTablesArgs &a, hipStream_t s) {
    if (a.R <= 256 && a.max_new <= kFusedTokens / 4) {
        hipLaunchKernelGGL((tables_scan_kernel<true, 256>), dim3(1), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    if (a.R <= kScanThreads && a.max_new <= kFusedTokens) {
        hipLaunchKernelGGL((tables_scan_kernel<true, kScanThreads>), dim3(1), dim3(kScanThreads), 0, s, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((tables_scan_kernel<false, kScanThreads>), dim3(1), dim3(kScanThreads), 0, s, a);
    const int64_t token_groups = ((int64_t)a.max_new + kFillThreads * kFillTokens - 1) / (kFillThreads * kFillTokens);
    const int64_t back_groups = ((int64_t)a.R + kFillThreads - 1) / kFillThreads;
    const dim3 grid((unsigned)(token_groups + back_groups));
    if (a.R <= kFillRequests) hipLaunchKernelGGL(tables_fill_kernel<true>, grid, dim3(kFillThreads), 0, s, a, (int32_t)token_groups);
    else hipLaunchKernelGGL(tables_fill_kernel<false>, grid, dim3(kFillThreads), 0, s, a, (int32_t)token_groups);
    return hipGetLastError();
}

hipError_t launch_kv_append(const KvAppendArgs &a, bool e4m3, hipStream_t s) {
    if (e4m3) {
        const int pieces = std::max(a.k_row, a.v ? a.v_row : 0);
        if (pieces <= 8) launch_e4m3<8, 1>(a, s);
        else if (pieces <= 16) launch_e4m3<16, 1>(a, s);
        else if (pieces <= 32) launch_e4m3<32, 1>(a, s);
        else launch_e4m3<64, 2>(a, s);             // latent rows: up to 72 pieces
        return hipGetLastError();
    }
    const uint32_t k_pieces = (uint32_t)a.heads * a.k_row, pieces = k_pieces + (a.v ? (uint32_t)a.heads * a.v_row : 0u);
    const int64_t groups = (a.T * pieces + 255) / 256;
    constexpr int64_t kMost = (1ll << 31) / 256;
    for (int64_t g = 0; g < groups; g += kMost)
        hipLaunchKernelGGL(append_copy_kernel, dim3((unsigned)std::min(kMost, groups - g)), dim3(256), 0, s, a, k_pieces, pieces, (uint32_t)g);
    return hipGetLastError();
}

}  // namespace craft
