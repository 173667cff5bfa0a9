// kv8_api.hip -- the C entry points of the batch plan and of the 8-bit paged K/V cache: host checks,
// then one launcher each.  See include/mg.h for the contract.
#include <math.h>

#include <atomic>

#include "../../include/mg.h"
#include "mg_kernels.h"

using namespace mg;

namespace {

bool dims_ok(int n_pages, int n_kv_heads, int head_dim) {
    return n_pages >= 1 && n_pages < (1 << 27) && n_kv_heads >= 1 && n_kv_heads <= 1024 &&
           (head_dim == 64 || head_dim == 128);
}
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// MG_OK, or why the cache is refused
mg_status cache_status(const mg_kv8_cache* c) {
    if (!c || !c->codes || !c->scales || !aligned(c->codes, 16) || !aligned(c->scales, 2)) return MG_ERR_ARG;
    return dims_ok(c->n_pages, c->n_kv_heads, c->head_dim) ? MG_OK : MG_ERR_SHAPE;
}
Kv8 view(const mg_kv8_cache* c) { return Kv8{c->codes, c->scales, c->n_pages, c->n_kv_heads, c->head_dim}; }
bool rows_ok(const mg_kv8_cache* c, const void* p, int64_t stride) {
    return aligned(p, 16) && stride % 8 == 0 && stride >= (int64_t)c->n_kv_heads * c->head_dim;
}
// n int32 values at p
struct Ints {
    const int32_t* p;
    size_t n;
    bool overlaps(const Ints& o) const {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
        return n && o.n && a < b + 4 * o.n && b < a + 4 * n;
    }
};
mg_status status_of(hipError_t e) { return e == hipSuccess ? MG_OK : MG_ERR_HIP; }

// compute units of the current device, looked up once a device (256 where that fails)
int cu_count() {
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
mg_status attn_args(const mg_kv8_cache* c, const mg_kv8_attn_args* g, Kv8AttnArgs* a) {
    const mg_status st = cache_status(c);
    if (st != MG_OK) return st;
    if (!g || g->n_rows < 0 || g->n_tokens < 0 || g->max_pages_per_row <= 0 || g->max_pages_per_row > (1 << 26))
        return MG_ERR_ARG;
    if (g->n_q_heads <= 0 || g->n_q_heads % c->n_kv_heads || g->n_q_heads / c->n_kv_heads > 16) return MG_ERR_SHAPE;
    if (g->max_new < 1 || g->max_len < 0 || g->window < 0) return MG_ERR_ARG;
    // (outside of this range their products with each other and with log2 e leave fp32's)
    const auto factor = [](float f) { return f >= 1e-15f && f <= 1e15f; };
    if ((g->scale != 0.0f && !factor(g->scale)) || (g->softcap != 0.0f && !factor(g->softcap))) return MG_ERR_ARG;
    const int64_t width = (int64_t)g->n_q_heads * c->head_dim;
    if (g->n_rows && g->n_tokens &&
        (!g->q || !g->out || !g->page_table || !g->lens || !aligned(g->q, 16) || !aligned(g->out, 16)))
        return MG_ERR_ARG;
    if (g->q_stride % 8 || g->q_stride < width || g->out_stride % 8 || g->out_stride < width) return MG_ERR_ARG;
    if (!g->cu_new && (g->n_tokens != g->n_rows || g->max_new != 1)) return MG_ERR_ARG;
    const int64_t cap = 16ll * g->max_pages_per_row;
    a->c = view(c);
    a->B = g->n_rows;
    a->T = g->n_tokens;
    a->Hq = g->n_q_heads;
    a->G = g->n_q_heads / c->n_kv_heads;
    a->max_new = g->max_new < g->n_tokens ? g->max_new : g->n_tokens;
    a->max_len = g->max_len && g->max_len < cap ? g->max_len : (int)cap;
    a->maxp = g->max_pages_per_row;
    a->window = g->window;
    a->scale = g->scale > 0.0f ? g->scale : (float)(1.0 / sqrt((double)c->head_dim));
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
    if (a->B && a->T && !kv8_attention_fits(*a)) return MG_ERR_ARG;
    return MG_OK;
}

}  // namespace

extern "C" {

size_t mg_kv8_code_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * 2 * 16 * head_dim : 0;
}

size_t mg_kv8_scale_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * 2 : 0;
}

mg_status mg_batch_plan(int B, int max_pages_per_row, const int32_t* ctx_len, const int32_t* n_new,
                        const int32_t* free_pages, const int32_t* n_free, int max_tokens, int32_t* page_table,
                        int32_t* cu_new, int32_t* lens, int32_t* admitted, int32_t* positions, int32_t* rows,
                        int32_t* slots, int32_t* n_left, void* stream) {
    if (B < 1 || B > PLAN_MAXB || max_pages_per_row < 1 || max_pages_per_row >= (1 << 27)) return MG_ERR_ARG;
    if (max_tokens < 0 || max_tokens > (1 << 30)) return MG_ERR_ARG;
    if (!ctx_len || !n_new || !free_pages || !n_free || !page_table || !cu_new || !lens || !admitted || !n_left)
        return MG_ERR_ARG;
    if (max_tokens && (!positions || !rows || !slots)) return MG_ERR_ARG;
    // blocks of the launch read the inputs while others write (of the free pages the host knows the first alone)
    const size_t rows_n = B, items = max_tokens;
    const Ints table{page_table, rows_n * max_pages_per_row};
    const Ints in[] = {{ctx_len, rows_n}, {n_new, rows_n}, {n_free, 1}, {free_pages, 1}, table};
    const Ints out[] = {{cu_new, rows_n + 1}, {lens, rows_n}, {admitted, rows_n}, {positions, items},
                        {rows, items},        {slots, items}, {n_left, 1}};
    for (const Ints& i : in)
        for (const Ints& o : out)
            if (i.overlaps(o)) return MG_ERR_ARG;
    for (int i = 0; i < 4; ++i)
        if (in[i].overlaps(table)) return MG_ERR_ARG;
    PlanArgs a{B,          max_pages_per_row, max_tokens, ctx_len, n_new,     free_pages, n_free, page_table,
               cu_new,     lens,              admitted,   positions, rows,    slots,      n_left};
    return status_of(launch_batch_plan(a, static_cast<hipStream_t>(stream)));
}

mg_status mg_kv8_append(const mg_kv8_cache* cache, int n_tokens, const uint16_t* k, int64_t k_stride,
                        const uint16_t* v, int64_t v_stride, const int32_t* slots, void* stream) {
    const mg_status st = cache_status(cache);
    if (st != MG_OK) return st;
    if (n_tokens < 0 || (int64_t)n_tokens * cache->n_kv_heads > KV8_MOST_PAIRS) return MG_ERR_ARG;
    if (n_tokens == 0) return MG_OK;
    if (!k || !v || !slots || !rows_ok(cache, k, k_stride) || !rows_ok(cache, v, v_stride)) return MG_ERR_ARG;
    return status_of(launch_kv8_append(view(cache), n_tokens, k, k_stride, v, v_stride, slots,
                                       static_cast<hipStream_t>(stream)));
}

mg_status mg_kv8_read(const mg_kv8_cache* cache, int n, const int32_t* slots, uint16_t* k, int64_t k_stride,
                      uint16_t* v, int64_t v_stride, void* stream) {
    const mg_status st = cache_status(cache);
    if (st != MG_OK) return st;
    if (n < 0 || (int64_t)n * cache->n_kv_heads > KV8_MOST_PAIRS) return MG_ERR_ARG;
    if (n == 0 || (!k && !v)) return MG_OK;
    if (!slots || (k && !rows_ok(cache, k, k_stride)) || (v && !rows_ok(cache, v, v_stride))) return MG_ERR_ARG;
    return status_of(launch_kv8_read(view(cache), n, slots, k, k_stride, v, v_stride,
                                     static_cast<hipStream_t>(stream)));
}

size_t mg_kv8_attention_workspace_bytes(const mg_kv8_cache* cache, const mg_kv8_attn_args* args) {
    Kv8AttnArgs a{};
    if (attn_args(cache, args, &a) != MG_OK || a.T == 0 || a.B == 0) return 0;
    return kv8_attention_ws_bytes(a);
}

mg_status mg_kv8_attention(const mg_kv8_cache* cache, const mg_kv8_attn_args* args, void* workspace,
                           size_t workspace_bytes, void* stream) {
    Kv8AttnArgs a{};
    const mg_status st = attn_args(cache, args, &a);
    if (st != MG_OK) return st;
    if (a.T == 0 || a.B == 0) return MG_OK;
    if (a.out == a.q) return MG_ERR_ARG;
    const size_t need = kv8_attention_ws_bytes(a);
    if (need && (!workspace || workspace_bytes < need)) return MG_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return MG_ERR_ARG;
    a.part = static_cast<float*>(workspace);
    return status_of(launch_kv8_attention(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
