// Entry points of the products (8-bit integers, grouped by expert): argument checks and launches.
#include "kernels.h"

namespace {

using namespace craft;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kInts = (int64_t)1 << 31;       // 32-bit indices stay below this
constexpr int64_t kFarthest = (int64_t)1 << 46;   // bytes from a matrix' start to its end
constexpr int64_t kMostRows = (int64_t)1 << 26;    // of a grouped product: tiles of groups that overlap stay countable
constexpr int32_t kMostCodes = 131071;            // of a contraction: products of two codes are at most 2^14, sums below 2^31
constexpr int64_t kLongestRow = (int64_t)1 << 23; // bytes of the contraction: 256 rows stay inside a 32-bit offset

inline int element_bytes(int32_t format) { return format == CRAFT_F32 ? 4 : format == CRAFT_BF16 ? 2 : 1; }

// rows of `row` bytes, `stride` elements of `es` bytes apart
bool rows_fit(int64_t rows, int64_t row, int64_t stride, int es) {
    if (stride <= 0 || stride > kFarthest / es || stride * es < row || (stride * es) % 16) return false;
    return rows <= 1 || stride * es <= kFarthest / rows;
}

// what both products share: sizes, x and the result
craft_status sizes(int32_t format, int32_t out_dtype, int64_t M, int32_t N, int32_t K, int64_t x_rows, int64_t x_stride,
                   int64_t out_stride, ProductArgs *a) {
    if (format != CRAFT_F32 && format != CRAFT_BF16 && format != CRAFT_I8) return CRAFT_EINVAL;
    if (out_dtype != CRAFT_F32 && out_dtype != CRAFT_BF16) return CRAFT_EINVAL;
    if (format != CRAFT_I8 && out_dtype != format) return CRAFT_EINVAL;
    const int es = element_bytes(format), os = element_bytes(out_dtype);
    if (M < 0 || M >= kInts || N <= 0 || N > (1 << 30) || K <= 0 || (int64_t)K * es >= kLongestRow || K % (16 / es)) return CRAFT_EINVAL;
    if (format == CRAFT_I8 && K > kMostCodes) return CRAFT_EINVAL;
    if (x_rows < 0 || x_rows >= kInts || !rows_fit(x_rows, (int64_t)K * es, x_stride, es)) return CRAFT_EINVAL;
    if (out_stride < N || out_stride > kFarthest / os || (M > 1 && out_stride * os > kFarthest / M)) return CRAFT_EINVAL;
    a->format = format;
    a->out_dtype = out_dtype;
    a->N = N;
    a->row_bytes = K * es;
    a->M = M;
    a->x_rows = x_rows;
    a->x_stride = x_stride * es;
    a->out_stride = out_stride;
    return CRAFT_OK;
}

bool operands(const void *x, const float *x_scale, void *out, ProductArgs *a) {
    if (!x || !aligned(x, 16) || !out || !aligned(out, element_bytes(a->out_dtype))) return false;
    if (a->format == CRAFT_I8 && (!x_scale || !aligned(x_scale, 4))) return false;
    a->x = static_cast<const unsigned char *>(x);
    a->x_scale = x_scale;
    a->out = out;
    a->out_whole = aligned(out, 4 * element_bytes(a->out_dtype)) && a->out_stride % 4 == 0;
    return true;
}

craft_status launched(hipError_t e) { return e == hipSuccess ? CRAFT_OK : CRAFT_EHIP; }

}  // namespace

extern "C" {

craft_status craft_quantize_i8(int32_t dtype, const void *x, int64_t x_stride, int64_t rows, int32_t K, int8_t *codes,
                               float *scale, void *stream) {
    if (dtype != CRAFT_F32 && dtype != CRAFT_BF16) return CRAFT_EINVAL;
    const int es = element_bytes(dtype);
    if (rows < 0 || rows >= ((int64_t)1 << 40) || K <= 0 || K % 16) return CRAFT_EINVAL;
    if (!rows_fit(rows, (int64_t)K * es, x_stride, es)) return CRAFT_EINVAL;
    if (rows == 0) return CRAFT_OK;
    if (!x || !aligned(x, 16) || !codes || !aligned(codes, 16) || !scale || !aligned(scale, 4)) return CRAFT_EINVAL;
    QuantizeI8Args a{};
    a.dtype = dtype;
    a.rows = rows;
    a.K = K;
    a.x_stride = x_stride * es;
    a.x = static_cast<const unsigned char *>(x);
    a.codes = codes;
    a.scale = scale;
    return launched(launch_quantize_i8(a, static_cast<hipStream_t>(stream)));
}

craft_status craft_matmul_i8(int64_t M, int32_t N, int32_t K, const int8_t *x, int64_t x_stride, const float *x_scale,
                             const int8_t *w, const float *w_scale, int32_t out_dtype, void *out, int64_t out_stride,
                             void *stream) {
    ProductArgs a{};
    const craft_status st = sizes(CRAFT_I8, out_dtype, M, N, K, M, x_stride, out_stride, &a);
    if (st != CRAFT_OK) return st;
    if (M == 0) return CRAFT_OK;
    if (!operands(x, x_scale, out, &a) || !w || !aligned(w, 16) || !w_scale || !aligned(w_scale, 4)) return CRAFT_EINVAL;
    a.G = 1;
    a.k = 1;
    a.w_one = reinterpret_cast<const unsigned char *>(w);
    a.w_one_scale = w_scale;
    a.num_cu = num_compute_units();
    return launched(launch_product(a, static_cast<hipStream_t>(stream)));
}

craft_status craft_grouped_matmul(const craft_grouped_matmul_args *g, void *stream) {
    if (!g) return CRAFT_EINVAL;
    ProductArgs a{};
    const craft_status st = sizes(g->format, g->out_dtype, g->M, g->N, g->K, g->src ? g->x_rows : g->M, g->x_stride, g->out_stride, &a);
    if (st != CRAFT_OK) return st;
    if (g->G <= 0 || g->G > kMostGroups || g->M > kMostRows) return CRAFT_EINVAL;
    if (g->src && (g->k <= 0 || !aligned(g->src, 4))) return CRAFT_EINVAL;
    if (g->M == 0) return CRAFT_OK;
    if (g->src && g->x_rows == 0) return CRAFT_EINVAL;         // places whose row is not there are read from row 0
    if (!operands(g->x, g->x_scale, g->out, &a)) return CRAFT_EINVAL;
    if (!g->off || !aligned(g->off, 4) || !g->w || !aligned(g->w, 8) || (g->w_up && !aligned(g->w_up, 8))) return CRAFT_EINVAL;
    if (g->format == CRAFT_I8) {
        if (!g->w_scale || !aligned(g->w_scale, 8) || (g->w_up && (!g->up_scale || !aligned(g->up_scale, 8)))) return CRAFT_EINVAL;
    }
    a.G = g->G;
    a.k = g->src ? g->k : 1;
    if (a.k > 1) {
        int bits = 1;                              // ceil(log2 k)
        while (((int64_t)1 << bits) < a.k) ++bits;
        a.k_magic = (uint32_t)((((uint64_t)1 << (31 + bits)) + (uint32_t)a.k - 1) / (uint32_t)a.k);
        a.k_shift = (uint32_t)(bits - 1);
    }
    a.src = g->src;
    a.off = g->off;
    a.w = reinterpret_cast<const unsigned char *const *>(g->w);
    a.up = reinterpret_cast<const unsigned char *const *>(g->w_up);
    a.w_scale = g->w_scale;
    a.up_scale = g->up_scale;
    a.num_cu = num_compute_units();
    return launched(launch_product(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
