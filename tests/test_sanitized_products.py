"""The host code of the products (product.cpp: argument checks, sizes, strides) under AddressSanitizer and
UndefinedBehaviorSanitizer, compiled by the host compiler with the launches replaced by checks of what they are given:
arguments from one end of their types to the other, most calls refused, every accepted one within the limits that the
kernels count on."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_28768_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "kernels.h"

using namespace craft;
static long launched[2];
#define WITHIN(x) do { if (!(x)) { std::printf("line %d: not %s\n", __LINE__, #x); std::exit(3); } } while (0)
static bool at16(const void *p) { return p && reinterpret_cast<uintptr_t>(p) % 16 == 0; }
// rows of `row` bytes every `stride` bytes end within 2^46 bytes
static bool rows_fit(int64_t rows, int64_t row, int64_t stride) {
    return row > 0 && row % 16 == 0 && stride >= row && stride % 16 == 0 && stride <= (1ll << 46) && (rows <= 1 || stride <= (1ll << 46) / rows);
}

int craft::num_compute_units() { return 256; }
hipError_t craft::launch_quantize_i8(const QuantizeI8Args &a, hipStream_t) {
    const int es = a.dtype == CRAFT_F32 ? 4 : 2;
    WITHIN(a.dtype == CRAFT_F32 || a.dtype == CRAFT_BF16);
    WITHIN(a.rows > 0 && a.rows < (1ll << 40) && a.K > 0 && a.K % 16 == 0 && at16(a.x) && at16(a.codes) && a.scale);
    WITHIN(rows_fit(a.rows, (int64_t)a.K * es, a.x_stride));
    ++launched[0];
    return hipSuccess;
}
hipError_t craft::launch_product(const ProductArgs &a, hipStream_t) {
    const int os = a.out_dtype == CRAFT_F32 ? 4 : 2;
    WITHIN(a.format == CRAFT_F32 || a.format == CRAFT_BF16 || a.format == CRAFT_I8);
    WITHIN(a.out_dtype == CRAFT_F32 || a.out_dtype == CRAFT_BF16);
    WITHIN(a.format == CRAFT_I8 || a.out_dtype == a.format);
    WITHIN(a.G >= 1 && a.G <= kMostGroups && a.N >= 1 && a.N <= (1 << 30) && a.k >= 1 && a.M > 0);
    WITHIN(a.off ? a.M <= (1ll << 26) : a.M < (1ll << 31));
    // 256 rows of a matrix inside a 32-bit offset, sums of codes inside 32 bits
    WITHIN(a.row_bytes > 0 && a.row_bytes % 16 == 0 && a.row_bytes < (1 << 23) && (a.format != CRAFT_I8 || a.row_bytes < 131072));
    WITHIN(a.x_rows > 0 && a.x_rows < (1ll << 31) && rows_fit(a.x_rows, a.row_bytes, a.x_stride) && at16(a.x) && a.out);
    WITHIN(a.src || a.x_rows == a.M);
    WITHIN(a.out_stride >= a.N && a.out_stride <= (1ll << 46) / os && (a.M <= 1 || a.out_stride * os <= (1ll << 46) / a.M));
    WITHIN(!a.out_whole || (reinterpret_cast<uintptr_t>(a.out) % (4 * os) == 0 && a.out_stride % 4 == 0));
    WITHIN(a.format != CRAFT_I8 || a.x_scale);
    if (a.off) WITHIN(a.w && (a.format != CRAFT_I8 || (a.w_scale && (!a.up || a.up_scale))));
    else WITHIN(!a.up && !a.src && a.G == 1 && at16(a.w_one) && a.w_one_scale);
    // the quotient by k as the kernels take it
    if (a.k > 1)
        for (uint32_t s : {0u, 1u, (uint32_t)a.k - 1, (uint32_t)a.k, 2u * a.k - 1, 0x7fffffffu, 0x7fffffffu / (uint32_t)a.k * a.k, 0x7fffffffu / (uint32_t)a.k * a.k - 1, 0x40000000u, 123456789u}) {
            s &= 0x7fffffffu;
            WITHIN((uint32_t)(((uint64_t)s * a.k_magic) >> 32) >> a.k_shift == s / (uint32_t)a.k);
        }
    ++launched[1];
    return hipSuccess;
}

static std::mt19937_64 rng(7);
// mostly something ordinary, otherwise from the ends of the type or of a limit
template <typename T> static T any(std::initializer_list<T> ordinary, int odds) {
    if (rng() % 100 >= (unsigned)odds) return ordinary.begin()[rng() % ordinary.size()];
    const int bits = 8 * sizeof(T) - 1;
    const int64_t most = bits == 63 ? INT64_MAX : INT32_MAX;
    switch (rng() % 6) {
    case 0: return (T)most;
    case 1: return (T)(-most - 1);
    case 2: return (T)((int64_t)(rng() % 5) - 2);
    case 3: return (T)(most - (int64_t)(rng() % 3000));
    case 4: return (T)((1ll << rng() % bits) - (int64_t)(rng() % 3) + 1);
    default: return (T)rng();
    }
}
template <typename T> static T *at(int odds) {
    if (rng() % 100 >= (unsigned)odds) return reinterpret_cast<T *>((uintptr_t)1 << 40);
    return reinterpret_cast<T *>(rng() % 2 ? 0 : ((uintptr_t)1 << 40) + rng() % 16);
}

int main() {
    for (long i = 0; i < 2000000; ++i) {
        const int odds = (int[]){0, 2, 5, 20}[rng() % 4];
        craft_quantize_i8(any<int32_t>({0, 1}, odds), at<void>(odds), any<int64_t>({64, 4096, 7168, 1 << 20}, odds), any<int64_t>({0, 1, 250, 1 << 20}, odds),
                          any<int32_t>({16, 64, 4096}, odds), at<int8_t>(odds), at<float>(odds), nullptr);
        craft_matmul_i8(any<int64_t>({0, 1, 61, 8192}, odds), any<int32_t>({1, 61, 4096}, odds), any<int32_t>({16, 64, 4096, 131056}, odds), at<int8_t>(odds),
                        any<int64_t>({131072, 1 << 20}, odds), at<float>(odds), at<int8_t>(odds), at<float>(odds), any<int32_t>({0, 1}, odds), at<void>(odds),
                        any<int64_t>({4096, 5000, 5001}, odds), nullptr);
        craft_grouped_matmul_args a;
        a.format = any<int32_t>({0, 1, 2}, odds);
        a.out_dtype = a.format == 2 ? any<int32_t>({0, 1}, odds) : any<int32_t>({a.format}, odds);
        a.G = any<int32_t>({1, 17, 1024}, odds);
        a.N = any<int32_t>({1, 61, 4096}, odds);
        a.K = any<int32_t>({16, 64, 4096}, odds);
        a.k = any<int32_t>({1, 2, 3, 6, 7, 8, 64, 1000003}, odds);
        a.M = any<int64_t>({0, 1, 4159, 1 << 26}, odds);
        a.x_rows = any<int64_t>({0, 1, 4096}, odds);
        a.x = at<void>(odds);
        a.x_stride = any<int64_t>({4096, 8192, 1 << 16}, odds);
        a.x_scale = at<float>(odds);
        a.src = rng() % 2 ? at<int32_t>(odds) : nullptr;
        a.off = at<int32_t>(odds);
        a.w = at<const void *>(odds);
        a.w_up = rng() % 2 ? at<const void *>(odds) : nullptr;
        a.w_scale = at<const float *>(odds);
        a.up_scale = at<const float *>(odds);
        a.out = at<void>(odds);
        a.out_stride = any<int64_t>({4096, 5000, 5001}, odds);
        craft_grouped_matmul(&a, nullptr);
    }
    std::printf("launched %ld %ld\n", launched[0], launched[1]);
    return launched[0] > 10000 && launched[1] > 10000 ? 0 : 4;
}
"""


def test_argument_checks_are_clean_under_asan_and_ubsan(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    exe = str(tmp_path / "driver")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           str(tmp_path / "driver.cpp"), os.path.join(CSRC, "product.cpp"), "-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="exitcode=66", UBSAN_OPTIONS="print_stacktrace=1"))
    assert res.returncode == 0, (res.stdout + res.stderr)[-3000:]
