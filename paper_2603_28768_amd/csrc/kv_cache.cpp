// Entry points of the paged key/value cache: argument checks, workspace layout, launches.
#include <cmath>

#include "kernels.h"

namespace {

using namespace craft;

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

constexpr int64_t kInts = (int64_t)1 << 31;       // 32-bit indices stay below this
constexpr int32_t kMostShared = 65536;            // query heads of a cache head: a launch has one workgroup or more for each 16 or 64
constexpr float kLog2e = 1.4426950408889634f;     // scores are powers of two in the kernels
constexpr int64_t kFarthest = (int64_t)1 << 46;   // bytes a stride may span

// log2 of a page size, -1 if it is none
int page_shift(int32_t page_size) {
    if (page_size <= 0 || page_size > 65536 || (page_size & (page_size - 1))) return -1;
    return __builtin_ctz((unsigned)page_size);
}

struct CacheView {
    int shift;
    int bytes;                     // of a stored element
    bool latent;
    int64_t k[3], v[3];            // strides of page, head, token in bytes
};

bool strides_in_bytes(const int64_t in[3], int bytes, int64_t out[3]) {
    for (int i = 0; i < 3; ++i) {
        if (in[i] <= 0 || in[i] > kFarthest / bytes) return false;
        out[i] = in[i] * bytes;
        if (out[i] % 16) return false;
    }
    return out[2] < ((int64_t)1 << 26);
}

craft_status view_of(const craft_kv_cache *c, CacheView *w) {
    if (!c) return CRAFT_EINVAL;
    if (c->format != CRAFT_KV_F32 && c->format != CRAFT_KV_BF16 && c->format != CRAFT_KV_E4M3) return CRAFT_EINVAL;
    w->bytes = c->format == CRAFT_KV_F32 ? 4 : c->format == CRAFT_KV_BF16 ? 2 : 1;
    w->latent = c->v == nullptr;
    w->shift = page_shift(c->page_size);
    const int unit = 16 / w->bytes;
    if (w->shift < 0 || c->pages <= 0 || c->pages >= kInts || c->pages * c->page_size >= kInts) return CRAFT_EINVAL;
    if (c->heads <= 0 || c->heads > 65536 || c->dk <= 0 || c->dv <= 0 || c->dk % unit || c->dv % unit) return CRAFT_EINVAL;
    if (w->latent ? (c->dv > c->dk || c->dk > 576 || c->dv > 512) : (c->dk > 256 || c->dv > 256)) return CRAFT_EINVAL;
    const int64_t k[3] = {c->k_page, c->k_head, c->k_token}, v[3] = {c->v_page, c->v_head, c->v_token};
    if (!c->k || !aligned(c->k, 16) || !strides_in_bytes(k, w->bytes, w->k)) return CRAFT_EINVAL;
    if (w->latent) {
        for (int i = 0; i < 3; ++i) w->v[i] = w->k[i];
    } else if (!aligned(c->v, 16) || !strides_in_bytes(v, w->bytes, w->v)) {
        return CRAFT_EINVAL;
    }
    if (c->format == CRAFT_KV_E4M3) {
        if (!c->k_scale || !aligned(c->k_scale, 16)) return CRAFT_EINVAL;
        if (!w->latent && (!c->v_scale || !aligned(c->v_scale, 16))) return CRAFT_EINVAL;
    }
    return CRAFT_OK;
}

craft_status check_tables(const craft_kv_tables_args *a) {
    if (!a || a->R < 0 || a->max_pages <= 0 || a->max_new < 0) return CRAFT_EINVAL;
    if (page_shift(a->page_size) < 0 || (int64_t)a->max_pages * a->page_size >= kInts) return CRAFT_EINVAL;
    if (a->pages <= 0 || a->pages >= kInts || a->pages * a->page_size >= kInts) return CRAFT_EINVAL;
    if (a->table_stride < a->max_pages || a->table_stride > kFarthest) return CRAFT_EINVAL;
    return CRAFT_OK;
}

size_t tables_bytes(int32_t R) { return 16 + 3 * round_up((size_t)R * 4, 16); }

craft_status attention_args(const craft_kv_cache *c, const craft_attention_args *a, AttentionArgs *out) {
    CacheView w;
    const craft_status st = view_of(c, &w);
    if (st != CRAFT_OK) return st;
    if (!a || a->R < 0 || a->Hq <= 0 || a->Hq % c->heads || (int64_t)a->R * a->Hq >= kInts) return CRAFT_EINVAL;
    if (a->Hq / c->heads > kMostShared) return CRAFT_EINVAL;
    // twice the longest request is still a 32-bit number
    if (a->max_pages <= 0 || (int64_t)a->max_pages * c->page_size > kInts / 2 || a->window < 0) return CRAFT_EINVAL;
    AttentionArgs o{};
    o.format = c->format;
    o.R = a->R;
    o.Hq = a->Hq;
    o.heads = c->heads;
    o.group = a->Hq / c->heads;
    o.dk = c->dk;
    o.dv = c->dv;
    o.max_pages = a->max_pages;
    o.window = a->window;
    o.shift = w.shift;
    o.k = static_cast<const unsigned char *>(c->k);
    o.v = static_cast<const unsigned char *>(w.latent ? c->k : c->v);
    o.k_page = w.k[0]; o.k_head = w.k[1]; o.k_token = w.k[2];
    o.v_page = w.v[0]; o.v_head = w.v[1]; o.v_token = w.v[2];
    o.k_scale = c->k_scale;
    o.v_scale = w.latent ? c->k_scale : c->v_scale;
    o.pages = c->pages;
    *out = o;
    return CRAFT_OK;
}

}  // namespace

extern "C" {

craft_status craft_kv_tables_workspace(const craft_kv_tables_args *args, size_t *bytes) {
    const craft_status st = check_tables(args);
    if (st != CRAFT_OK || !bytes) return CRAFT_EINVAL;
    *bytes = tables_bytes(args->R);
    return CRAFT_OK;
}

craft_status craft_kv_tables(const craft_kv_tables_args *a, void *stream) {
    const craft_status st = check_tables(a);
    if (st != CRAFT_OK) return st;
    if (a->R > 0 && (!a->add || !a->lens || !a->table || !a->lens_out || !aligned(a->add, 4) || !aligned(a->lens, 4) ||
                     !aligned(a->table, 4) || !aligned(a->lens_out, 4)))
        return CRAFT_EINVAL;
    if (!a->ring || !a->pool || !a->pool_out || !a->token_off || !aligned(a->ring, 4) || !aligned(a->pool, 8) ||
        !aligned(a->pool_out, 8) || !aligned(a->token_off, 4))
        return CRAFT_EINVAL;
    if (a->max_new > 0 && (!a->slots || !aligned(a->slots, 4))) return CRAFT_EINVAL;
    if (a->positions && !aligned(a->positions, 4)) return CRAFT_EINVAL;
    if (!a->workspace || !aligned(a->workspace, 16)) return CRAFT_EINVAL;
    if (a->workspace_bytes < tables_bytes(a->R)) return CRAFT_EWORKSPACE;
    KvTablesArgs k{};
    k.R = a->R;
    k.max_pages = a->max_pages;
    k.max_new = a->max_new;
    k.shift = page_shift(a->page_size);
    k.pages = a->pages;
    k.table_stride = a->table_stride;
    k.add = a->add;
    k.lens = a->lens;
    k.table = a->table;
    k.ring = a->ring;
    k.pool = a->pool;
    k.lens_out = a->lens_out;
    k.pool_out = a->pool_out;
    k.token_off = a->token_off;
    k.slots = a->slots;
    k.positions = a->positions;
    const size_t part = round_up((size_t)a->R * 4, 16) / 4;
    k.ws_ctrl = static_cast<int32_t *>(a->workspace);
    k.ws_len = k.ws_ctrl + 4;
    k.ws_page = k.ws_len + part;
    k.ws_back = k.ws_page + part;
    return launch_kv_tables(k, static_cast<hipStream_t>(stream)) == hipSuccess ? CRAFT_OK : CRAFT_EHIP;
}

craft_status craft_kv_append(const craft_kv_cache *cache, int64_t T, const void *k, int64_t k_stride, const void *v,
                             int64_t v_stride, const int32_t *slots, void *stream) {
    CacheView w;
    const craft_status st = view_of(cache, &w);
    if (st != CRAFT_OK) return st;
    if (T < 0 || T >= ((int64_t)1 << 40)) return CRAFT_EINVAL;
    if (T == 0) return CRAFT_OK;
    const int es = cache->format == CRAFT_KV_F32 ? 4 : 2;      // of the new rows
    const int64_t k_row = (int64_t)cache->heads * cache->dk, v_row = (int64_t)cache->heads * cache->dv;
    if (!k || !aligned(k, 16) || k_stride < k_row || k_stride > kFarthest || k_stride * es % 16) return CRAFT_EINVAL;
    if (!w.latent && (!v || !aligned(v, 16) || v_stride < v_row || v_stride > kFarthest || v_stride * es % 16)) return CRAFT_EINVAL;
    if (!slots || !aligned(slots, 4)) return CRAFT_EINVAL;
    KvAppendArgs a{};
    a.T = T;
    a.heads = cache->heads;
    a.k_row = cache->dk * es / 16;
    a.v_row = cache->dv * es / 16;
    a.k = static_cast<const unsigned char *>(k);
    a.v = w.latent ? nullptr : static_cast<const unsigned char *>(v);
    a.k_stride = k_stride * es;
    a.v_stride = w.latent ? 0 : v_stride * es;     // ignored for latent rows, whatever it is
    a.slots = slots;
    a.slots_total = cache->pages * cache->page_size;
    a.shift = w.shift;
    a.ck = static_cast<unsigned char *>(cache->k);
    a.cv = static_cast<unsigned char *>(cache->v);
    a.ck_page = w.k[0]; a.ck_head = w.k[1]; a.ck_token = w.k[2];
    a.cv_page = w.v[0]; a.cv_head = w.v[1]; a.cv_token = w.v[2];
    a.k_scale = cache->k_scale;
    a.v_scale = cache->v_scale;
    return launch_kv_append(a, cache->format == CRAFT_KV_E4M3, static_cast<hipStream_t>(stream)) == hipSuccess ? CRAFT_OK : CRAFT_EHIP;
}

craft_status craft_decode_attention_workspace(const craft_kv_cache *cache, const craft_attention_args *args, size_t *bytes) {
    AttentionArgs a;
    const craft_status st = attention_args(cache, args, &a);
    if (st != CRAFT_OK) return st;
    if (!bytes) return CRAFT_EINVAL;
    *bytes = attention_workspace(a, num_compute_units());
    return CRAFT_OK;
}

craft_status craft_decode_attention(const craft_kv_cache *cache, const craft_attention_args *args, void *stream) {
    AttentionArgs a;
    const craft_status st = attention_args(cache, args, &a);
    if (st != CRAFT_OK) return st;
    if (!std::isfinite(args->scale * kLog2e)) return CRAFT_EINVAL;
    if (a.R == 0) return CRAFT_OK;
    const int es = cache->format == CRAFT_KV_F32 ? 4 : 2;
    if (!args->q || !aligned(args->q, 16) || args->q_stride <= 0 || args->q_head_stride < cache->dk) return CRAFT_EINVAL;
    if (args->q_stride > kFarthest || args->q_head_stride >= ((int64_t)1 << 24) || args->q_stride * es % 16 || args->q_head_stride * es % 16)
        return CRAFT_EINVAL;
    if (!args->lens || !args->table || !args->out || !aligned(args->lens, 4) || !aligned(args->table, 4) || !aligned(args->out, 16))
        return CRAFT_EINVAL;
    if (args->lse && !aligned(args->lse, 4)) return CRAFT_EINVAL;
    if (args->table_stride < args->max_pages || args->table_stride > kFarthest) return CRAFT_EINVAL;
    if (!args->workspace || !aligned(args->workspace, 16)) return CRAFT_EINVAL;
    const int32_t cus = num_compute_units();
    if (args->workspace_bytes < attention_workspace(a, cus)) return CRAFT_EWORKSPACE;
    a.q = args->q;
    a.q_stride = args->q_stride;
    a.q_head = args->q_head_stride;
    a.lens = args->lens;
    a.table = args->table;
    a.table_stride = args->table_stride;
    a.scale_log2 = args->scale * kLog2e;
    a.out = args->out;
    a.lse = args->lse;
    a.workers = attention_workers(a, cus);
    a.counters = static_cast<int32_t *>(args->workspace);
    a.part = reinterpret_cast<float *>(static_cast<unsigned char *>(args->workspace) + attention_counters_bytes());
    return launch_decode_attention(a, static_cast<hipStream_t>(stream)) == hipSuccess ? CRAFT_OK : CRAFT_EHIP;
}

}  // extern "C"
