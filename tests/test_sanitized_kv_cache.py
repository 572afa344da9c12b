"""The host code of the paged cache (kv_cache.cpp: argument checks, sizes, strides) under AddressSanitizer and
UndefinedBehaviorSanitizer, compiled by the host compiler with the launches replaced by checks of what they are given:
arguments from one end of their types to the other, most calls refused, every accepted one within the limits that the
kernels count on."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2603_28768_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include "kernels.h"

using namespace craft;
static long launched[3];
#define WITHIN(x) do { if (!(x)) { std::printf("line %d: not %s\n", __LINE__, #x); std::exit(3); } } while (0)

static bool span(int64_t s) { return s > 0 && s % 16 == 0 && s <= (1ll << 46); }

int craft::num_compute_units() { return 256; }
size_t craft::attention_counters_bytes() { return CRAFT_ATTENTION_COUNTER_BYTES; }
static void check_shape(const AttentionArgs &a) {
    WITHIN(a.R >= 0 && a.Hq > 0 && a.heads > 0 && a.group > 0 && (int64_t)a.heads * a.group == a.Hq);
    WITHIN((int64_t)a.R * a.Hq < (1ll << 31) && a.group <= 65536);
    // longer rows than 256 are latent ones
    WITHIN(a.dk > 0 && a.dv > 0 && ((a.dk <= 256 && a.dv <= 256) || (a.k == a.v && a.dk <= 576 && a.dv <= 512 && a.dv <= a.dk)));
    WITHIN(a.shift >= 0 && a.shift <= 16 && a.max_pages > 0 && ((int64_t)a.max_pages << a.shift) <= (1ll << 30) && a.window >= 0);
    WITHIN(a.pages > 0 && (a.pages << a.shift) < (1ll << 31));
    WITHIN(span(a.k_page) && span(a.k_head) && span(a.k_token) && a.k_token < (1 << 26));
    WITHIN(span(a.v_page) && span(a.v_head) && span(a.v_token) && a.v_token < (1 << 26));
    WITHIN(a.format != CRAFT_KV_E4M3 || (a.k_scale && a.v_scale));
}
int32_t craft::attention_workers(const AttentionArgs &a, int32_t) { check_shape(a); return 256; }
size_t craft::attention_workspace(const AttentionArgs &a, int32_t) { check_shape(a); return 1 << 20; }
hipError_t craft::launch_decode_attention(const AttentionArgs &a, hipStream_t) {
    check_shape(a);
    const int es = a.format == CRAFT_KV_F32 ? 4 : 2;
    WITHIN(a.R > 0 && a.q && a.lens && a.table && a.out && a.counters && a.part);
    WITHIN(a.q_stride > 0 && a.q_stride * es % 16 == 0 && a.q_head >= a.dk && a.q_head < (1 << 24) && a.q_head * es % 16 == 0);
    WITHIN(a.table_stride >= a.max_pages && a.table_stride <= (1ll << 46) && std::isfinite(a.scale_log2));
    ++launched[0];
    return hipSuccess;
}
hipError_t craft::launch_kv_tables(const KvTablesArgs &a, hipStream_t) {
    WITHIN(a.R >= 0 && a.max_pages > 0 && a.max_new >= 0 && a.shift >= 0 && a.shift <= 16);
    WITHIN(((int64_t)a.max_pages << a.shift) < (1ll << 31) && a.pages > 0 && (a.pages << a.shift) < (1ll << 31));
    WITHIN(a.table_stride >= a.max_pages && a.table_stride <= (1ll << 46));
    WITHIN(a.R == 0 || (a.add && a.lens && a.table && a.lens_out));
    WITHIN(a.ring && a.pool && a.pool_out && a.token_off && (a.max_new == 0 || a.slots));
    // the workspace's parts follow one another, each with room for all requests
    WITHIN(a.ws_len - a.ws_ctrl == 4 && a.ws_page - a.ws_len >= a.R && a.ws_back - a.ws_page >= a.R);
    ++launched[1];
    return hipSuccess;
}
hipError_t craft::launch_kv_append(const KvAppendArgs &a, bool e4m3, hipStream_t) {
    WITHIN(a.T > 0 && a.T < (1ll << 40) && a.heads > 0 && a.heads <= 65536 && a.k && a.slots && a.k_row > 0 && a.k_row <= 144);
    WITHIN(!a.v || (a.v_row > 0 && a.v_row <= 64));
    WITHIN(a.k_stride >= 16ll * a.heads * a.k_row && a.k_stride % 16 == 0 && (!a.v || (a.v_stride >= 16ll * a.heads * a.v_row && a.v_stride % 16 == 0)));
    WITHIN(a.slots_total > 0 && a.slots_total < (1ll << 31) && span(a.ck_page) && span(a.ck_head) && span(a.ck_token));
    WITHIN(!a.v || (a.cv && span(a.cv_page) && span(a.cv_head) && span(a.cv_token)));
    WITHIN(!e4m3 || (a.k_scale && (!a.v || a.v_scale)));
    ++launched[2];
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
        craft_kv_cache c;
        c.format = any<int32_t>({0, 1, 2}, odds);
        c.page_size = any<int32_t>({1, 8, 16, 64, 65536}, odds);
        c.pages = any<int64_t>({1, 100, 5000}, odds);
        c.heads = any<int32_t>({1, 2, 8, 65536}, odds);
        c.dk = any<int32_t>({16, 64, 128, 256}, odds);
        c.dv = any<int32_t>({16, 64, 128}, odds);
        c.k = at<void>(odds);
        c.v = rng() % 3 ? at<void>(odds) : nullptr;
        if (!c.v && rng() % 2) { c.dk = 576; c.dv = 512; }
        c.k_scale = at<float>(odds);
        c.v_scale = at<float>(odds);
        for (int64_t *s : {&c.k_page, &c.k_head, &c.k_token, &c.v_page, &c.v_head, &c.v_token}) *s = any<int64_t>({16, 64, 128, 4096, 1ll << 20}, odds);
        craft_attention_args a;
        a.R = any<int32_t>({0, 1, 7, 250}, odds);
        a.Hq = any<int32_t>({c.heads > 0 && c.heads <= 65536 ? c.heads : 8, c.heads > 0 && c.heads <= 65536 ? 16 * c.heads : 8, 64}, odds);
        a.max_pages = any<int32_t>({1, 10, 500, 16384}, odds);
        a.window = any<int32_t>({0, 1, 4096}, odds);
        a.scale = odds && rng() % 20 == 0 ? (float[]){3e38f, -3e38f, INFINITY, NAN, 0.0f}[rng() % 5] : 0.1f;
        a.q = at<void>(odds);
        a.q_stride = any<int64_t>({8192, 1ll << 30}, odds);
        a.q_head_stride = any<int64_t>({576, 1024}, odds);
        a.lens = at<int32_t>(odds);
        a.table = at<int32_t>(odds);
        a.table_stride = any<int64_t>({16384, 20000}, odds);
        a.out = at<void>(odds);
        a.lse = at<float>(odds);
        a.workspace = at<void>(odds);
        a.workspace_bytes = rng() % 10 ? (size_t)1 << 20 : rng() % ((size_t)2 << 20);
        size_t n = 0;
        craft_decode_attention_workspace(&c, &a, &n);
        craft_decode_attention(&c, &a, nullptr);
        craft_kv_append(&c, any<int64_t>({0, 1, 5000}, odds), at<void>(odds), any<int64_t>({1ll << 26, 4096}, odds), at<void>(odds),
                        any<int64_t>({1ll << 26, 4096}, odds), at<int32_t>(odds), nullptr);
        craft_kv_tables_args t;
        t.R = any<int32_t>({0, 1, 300, 5000}, odds);
        t.max_pages = any<int32_t>({1, 10, 500}, odds);
        t.page_size = c.page_size;
        t.max_new = any<int32_t>({0, 1, 10000}, odds);
        t.pages = c.pages;
        t.table_stride = any<int64_t>({500, 512}, odds);
        t.add = at<int32_t>(odds);
        t.lens = at<int32_t>(odds);
        t.table = at<int32_t>(odds);
        t.ring = at<int32_t>(odds);
        t.pool = at<int64_t>(odds);
        t.lens_out = at<int32_t>(odds);
        t.pool_out = at<int64_t>(odds);
        t.token_off = at<int32_t>(odds);
        t.slots = at<int32_t>(odds);
        t.positions = at<int32_t>(odds);
        t.workspace = at<void>(odds);
        t.workspace_bytes = rng() % 10 ? (size_t)1 << 36 : rng() % 100000;
        craft_kv_tables_workspace(&t, &n);
        craft_kv_tables(&t, nullptr);
    }
    std::printf("launched %ld %ld %ld\n", launched[0], launched[1], launched[2]);
    return launched[0] > 10000 && launched[1] > 10000 && launched[2] > 10000 ? 0 : 4;
}
"""


def test_argument_checks_are_clean_under_asan_and_ubsan(tmp_path):
    (tmp_path / "driver.cpp").write_text(DRIVER)
    exe = str(tmp_path / "driver")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                           str(tmp_path / "driver.cpp"), os.path.join(CSRC, "kv_cache.cpp"), "-o", exe])
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="exitcode=66", UBSAN_OPTIONS="print_stacktrace=1"))
    assert res.returncode == 0, (res.stdout + res.stderr)[-3000:]
