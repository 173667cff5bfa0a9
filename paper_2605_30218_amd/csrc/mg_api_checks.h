// mg_api_checks.h -- host checks that the entry points of the batch plan, the paged caches and the log probabilities share.
#pragma once
#include <math.h>

#include <atomic>

#include "../../include/mg.h"
#include "mg_kernels.h"

namespace mg {

inline bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// dimensions of a paged cache
inline bool cache_dims_ok(int n_pages, int n_kv_heads, int head_dim) {
    return n_pages >= 1 && n_pages < (1 << 27) && n_kv_heads >= 1 && n_kv_heads <= 1024 &&
           (head_dim == 64 || head_dim == 128);
}
// rows of `width` bf16 values at p
inline bool rows_ok(const void* p, int64_t stride, int64_t width) { return aligned(p, 16) && stride % 8 == 0 && stride >= width; }
// n int32 values at p
struct Ints {
    const int32_t* p;
    size_t n;
    bool overlaps(const Ints& o) const {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
        return n && o.n && a < b + 4 * o.n && b < a + 4 * n;
    }
};
inline mg_status status_of(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_HIP; }

// compute units of the current device, looked up once a device (256 where that fails)
inline int cu_count() {
    constexpr int MAX_DEVICES = 64;
    static std::atomic<int> known[MAX_DEVICES];
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return 256;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) return 256;
        known[dev].store(n, std::memory_order_relaxed);
    }
    return n;
}

// the checked arguments of an attention call as the kernels take them
// (c: a cache that was found sound; fits: whether the cache's launches are within the grid limits)
inline mg_status attn_args(const Kv8& c, const mg_kv8_attn_args* g, bool (*fits)(const Kv8AttnArgs&), Kv8AttnArgs* a) {
    if (!g || g->n_rows < 0 || g->n_tokens < 0 || g->max_pages_per_row <= 0 || g->max_pages_per_row > (1 << 26))
        return MG_ERR_ARG;
    if (g->n_q_heads <= 0 || g->n_q_heads % c.Hkv || g->n_q_heads / c.Hkv > 16) return MG_ERR_SHAPE;
    if (g->max_new < 1 || g->max_len < 0 || g->window < 0) return MG_ERR_ARG;
    // (outside of this range their products with each other and with log2 e leave fp32's)
    const auto factor = [](float f) { return f >= 1e-15f && f <= 1e15f; };
    if ((g->scale != 0.0f && !factor(g->scale)) || (g->softcap != 0.0f && !factor(g->softcap))) return MG_ERR_ARG;
    const int64_t width = (int64_t)g->n_q_heads * c.hd;
    if (g->n_rows && g->n_tokens &&
        (!g->q || !g->out || !g->page_table || !g->lens || !aligned(g->q, 16) || !aligned(g->out, 16)))
        return MG_ERR_ARG;
    if (g->q_stride % 8 || g->q_stride < width || g->out_stride % 8 || g->out_stride < width) return MG_ERR_ARG;
    if (!g->cu_new && (g->n_tokens != g->n_rows || g->max_new != 1)) return MG_ERR_ARG;
    const int64_t cap = 16ll * g->max_pages_per_row;
    a->c = c;
    a->B = g->n_rows;
    a->T = g->n_tokens;
    a->Hq = g->n_q_heads;
    a->G = g->n_q_heads / c.Hkv;
    a->max_new = g->max_new < g->n_tokens ? g->max_new : g->n_tokens;
    a->max_len = g->max_len && g->max_len < cap ? g->max_len : (int)cap;
    a->maxp = g->max_pages_per_row;
    a->window = g->window;
    a->scale = g->scale > 0.0f ? g->scale : (float)(1.0 / sqrt((double)c.hd));
    a->cap = g->softcap;
    a->inv_cap = g->softcap > 0.0f ? 1.0f / g->softcap : 0.0f;
    a->q = g->q;
    a->out = g->out;
    a->q_stride = g->q_stride;
    a->out_stride = g->out_stride;
    a->page_table = g->page_table;
    a->lens = g->lens;
    a->cu_new = g->cu_new;
    a->n_cu = cu_count();
    a->part = nullptr;
    if (a->B && a->T && !fits(*a)) return MG_ERR_ARG;
    return MG_OK;
}

}  // namespace mg
