// What the kernels of the attention of one new token share: the cut of the work into runs, and the running sums
// of a head as the matrix instructions leave them.
#pragma once

#include "ffn_common.h"
#include "shares.h"

namespace craft {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kUnit = 32;                          // tokens
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

static __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const unsigned char *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(p), 0, bytes, 0x00027000);
}
// Values are read once, whole lines at a time: streaming loads.  Keys are read 64 bytes of a row at a time, and the
// L1 keeps a line until its other half is asked for.  Two requests of 100001 and 131072 tokens, 8 heads of 128 in bf16:
// 184 us with no streaming loads, 166 with both, 170 (and with one workgroup per CU 159, 165) with values only.
constexpr int kStreaming = 2;
template <int W> struct Words;
template <> struct Words<4> {
    typedef u32x4_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kStreaming); }
};
template <> struct Words<2> {
    typedef u32x2_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kStreaming); }
};
template <> struct Words<1> {
    typedef uint32_t type;
    static __device__ __forceinline__ type load(__amdgpu_buffer_rsrc_t r, uint32_t off) { return __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, kStreaming); }
};
template <int W> __device__ __forceinline__ uint32_t word(const typename Words<W>::type &x, int i) { return x[i]; }
template <> __device__ __forceinline__ uint32_t word<1>(const uint32_t &x, int) { return x; }

// The same in every lane of the wave: kept in scalar registers.
static __device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
static __device__ __forceinline__ int64_t uniform(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)(x >> 32)) << 32 | (uint32_t)uniform((int32_t)x));
}

// Reductions over the four lanes that hold a head (lane & 15): rows of 16 lanes change places, odd ones of the one
// copy with even ones of the other, then halves of the wave.
static __device__ __forceinline__ float max_of_head(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
static __device__ __forceinline__ float sum_of_head(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t v = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
static __device__ __forceinline__ uint32_t perm(uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); }

static __device__ __forceinline__ int32_t length_of(const AttentionArgs &a, int32_t r) {
    return min(max(a.lens[r], 0), a.max_pages << a.shift);
}
static __device__ __forceinline__ int32_t first_of(const AttentionArgs &a, int32_t len) { return a.window > 0 ? max(len - a.window, 0) : 0; }
static __device__ __forceinline__ int32_t units_of(const AttentionArgs &a, int32_t len) {
    // an empty request is one unit without tokens, so that somebody writes its zeros
    return max(1, (len + kUnit - 1) / kUnit - first_of(a, len) / kUnit);
}

// The list of items cut into n runs.  Lengths in units, an item's own cost included.
struct Runs {
    int64_t total, each;   // the first `more` runs are one longer than `each`
    int32_t n, more;
    // at most `most` runs, of `least` or more where there is little to do
    __device__ __forceinline__ void cut(int64_t t, int32_t most, int32_t least) {
        total = t;
        n = (int32_t)min((int64_t)most, (t + least - 1) / least);
        if (t >> 32) {
            each = t / n;
        } else {
            each = (uint32_t)t / (uint32_t)n;
        }
        more = (int32_t)(t - each * n);
    }
    __device__ __forceinline__ int64_t start(int32_t w) const { return each * w + min(w, more); }
    __device__ __forceinline__ int32_t of(int64_t at) const {      // the run that holds place `at`
        const int64_t longer = (each + 1) * more, in = at < longer ? at : at - longer, of = at < longer ? each + 1 : each;
        return (at < longer ? 0 : more) + (total >> 32 ? (int32_t)(in / of) : (int32_t)((uint32_t)in / (uint32_t)of));
    }
};

// The request in which each wave's run starts, and the cost in front of it.
struct Start {
    int64_t before;
    int32_t request, len;
};
// per_request: items of a request, each of which costs item_cost beside its units.  The workgroup has COUNT runs,
// from `rank` on; a wave gets the start of the run of its number (of the only one).
template <int WAVES, int COUNT>
static __device__ __forceinline__ Start find_start(const AttentionArgs &a, int32_t per_request, int32_t item_cost, int32_t most, int32_t least, int32_t rank, Runs &runs) {
    __shared__ int64_t wave_sum[WAVES];
    __shared__ Start found[COUNT];
    constexpr int kThreads = 64 * WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t per = share_of<kThreads>(a.R);
    const int64_t r0 = min((int64_t)a.R, (int64_t)tid * per), r1 = min((int64_t)a.R, r0 + per);
    int64_t sum = 0;
    int32_t len = 0;                               // of the last request: of the only one, up to kThreads requests
    for (int64_t r = r0; r < r1; ++r) {
        len = length_of(a, (int32_t)r);
        sum += units_of(a, len) + item_cost;
    }
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
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += wave_sum[w];
        total += wave_sum[w];
    }
    runs.cut(uniform(total), most, least);
#pragma unroll
    for (int w = 0; w < COUNT; ++w) {
        const int64_t at = runs.start(rank + w);
        if (rank + w < runs.n && at >= before && at < before + sum) {
            int64_t b = before;
            int32_t r = (int32_t)r0;
            for (;; ++r) {
                if (per > 1) len = length_of(a, r);
                const int64_t u = (int64_t)(units_of(a, len) + item_cost) * per_request;
                if (at < b + u) break;
                b += u;
            }
            found[w] = {b, r, len};
        }
    }
    __syncthreads();
    const Start &mine = found[COUNT > 1 ? wave : 0];
    return {uniform(mine.before), uniform(mine.request), uniform(mine.len)};
}

// How far a running maximum may lag behind the scores, in powers of two: weights up to 256 are as exact as weights
// up to 1, and the sums are multiplied only when the maximum has grown by that much, which after the first units it
// hardly ever does.
constexpr float kSlack = 8.0f;

// Running maximum (or nearly), sum of weights and weighted sum of some tokens of an item, as a wave holds them: lane (head, g)
// has the sum of the weights of its own tokens only, the rest is whole.
template <int NV, int CE, bool F32> struct Sums {
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
    // Scores up to `top` come next: returns what to take from them.
    __device__ __forceinline__ float raise(float top) {
        if (__any(top > m + kSlack)) {
            const float up = fmaxf(m, top);
            scale(up == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - up));
            m = up;
        }
        return m == -INFINITY ? 0.0f : m;
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
    // The same for other workgroups, which may run on another XCD: stores that go through this one's L2 and loads
    // that go past theirs (device scope), 16 bytes at a time.  With fences instead, which write back or invalidate
    // the whole L2 of an XCD, 64 requests of 1 to 16384 tokens took 298 us, not 92.
    static constexpr int kDevice = 16;
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t sums_at(const float *p) { return rows_of(reinterpret_cast<const unsigned char *>(p), kFloats * 4); }
    __device__ __forceinline__ void put_out(float *to, int lane) const {
        const __amdgpu_buffer_rsrc_t rs = sums_at(to);
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, acc[c][e]), rs, (uint32_t)((c * CE + e) * 64 + lane) * 16, 0, kDevice);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(m), rs, (uint32_t)(NV * CE * 256 + lane) * 4, 0, kDevice);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(l), rs, (uint32_t)(NV * CE * 256 + 64 + lane) * 4, 0, kDevice);
    }
    __device__ __forceinline__ void add_from(const float *from, int lane) {
        const __amdgpu_buffer_rsrc_t rs = sums_at(from);
        const float om = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (uint32_t)(NV * CE * 256 + lane) * 4, 0, kDevice));
        const float ol = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (uint32_t)(NV * CE * 256 + 64 + lane) * 4, 0, kDevice));
        join(om, ol, [&](int c, int e) {
            return __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (uint32_t)((c * CE + e) * 64 + lane) * 16, 0, kDevice));
        });
    }
    __device__ __forceinline__ void add(const float *from, int lane) {
        join(from[NV * CE * 256 + lane], from[NV * CE * 256 + 64 + lane],
             [&](int c, int e) { return *reinterpret_cast<const f32x4_t *>(from + ((c * CE + e) * 64 + lane) * 4); });
    }
    template <typename F> __device__ __forceinline__ void join(float om, float ol, F acc_of) {
        const float up = fmaxf(m, om);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - up), of = om == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(om - up);
        m = up;
        l = l * f + ol * of;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < CE; ++e) {
                const f32x4_t x = acc_of(c, e);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[c][e][i] = acc[c][e][i] * f + x[i] * of;
                // no more than eight pieces on their way: registers
                if ((c * CE + e) % 8 == 7) __builtin_amdgcn_sched_barrier(0);
            }
    }
    // Row i of tile (c, e) is column ((c0 + c) 16 + 4 g + i) CE + e: CE neighbouring columns of the output per (c, i).
    __device__ __forceinline__ void write(const AttentionArgs &a, int32_t r, int32_t head0, int32_t n_heads, int lane, int c0 = 0) const {
        const int col = lane & 15, g = lane >> 4;
        const float sum = sum_of_head(l);
        if (col >= n_heads) return;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const int64_t head = (int64_t)r * a.Hq + head0 + col;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = ((c0 + c) * 16 + 4 * g + i) * CE;
                if (d >= a.dv) continue;
                if constexpr (CE == 1) {           // rows, and columns of the output, 4 g .. 4 g + 3 together
                    if (i == 0) {
                        const f32x4_t x = acc[c][0] * inv;
                        *reinterpret_cast<u32x2_t *>(static_cast<unsigned char *>(a.out) + (head * a.dv + d) * 2) = (u32x2_t){bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
                    }
                } else if constexpr (F32) {
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
        if (c0 == 0 && g == 0 && a.lse) a.lse[head] = sum == 0.0f ? -INFINITY : (m + __log2f(sum)) * 0.6931471805599453f;
    }
};

// An item in the list, and its request and number there.
struct Place {
    int64_t begin, end;
    int32_t request, item;
};
// An item that several workgroups have parts of, the first of them with its first unit.
struct Cut {
    Place item;
    int32_t mine;
};
constexpr int kJoin = 16;                          // parts joined by one workgroup
constexpr int kCounters = 4096;                    // of a kind: most workgroups of a launch

// One lane arrives at the counter for its workgroup, when the stores of all of it have been made (put_out: they are
// then where every XCD sees them).  Whether it was the last of `of`, which leaves the counter as it was found, at zero.
static __device__ __forceinline__ bool last_to_arrive(int32_t *counter, int32_t of, int32_t *shared) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        *shared = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
        if (*shared) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    const bool last = *shared != 0;
    __syncthreads();
    return last;
}

}  // namespace craft
