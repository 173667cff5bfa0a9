// kv8_api.hip -- the C entry points of the batch plan and of the 8-bit paged K/V cache: host checks,
// then one launcher each.  See include/mg.h for the contract.
#include "mg_api_checks.h"

using namespace mg;

namespace {

// MG_OK, or why the cache is refused
mg_status cache_status(const mg_kv8_cache* c) {
    if (!c || !c->codes || !c->scales || !aligned(c->codes, 16) || !aligned(c->scales, 2)) return MG_ERR_ARG;
    return cache_dims_ok(c->n_pages, c->n_kv_heads, c->head_dim) ? MG_OK : MG_ERR_SHAPE;
}
Kv8 view(const mg_kv8_cache* c) { return Kv8{c->codes, c->scales, c->n_pages, c->n_kv_heads, c->head_dim}; }
bool rows_ok(const mg_kv8_cache* c, const void* p, int64_t stride) {
    return mg::rows_ok(p, stride, (int64_t)c->n_kv_heads * c->head_dim);
}
// the checked arguments of an attention call as the kernels take them
mg_status attn_args(const mg_kv8_cache* c, const mg_kv8_attn_args* g, Kv8AttnArgs* a) {
    const mg_status st = cache_status(c);
    return st == MG_OK ? attn_args(view(c), g, kv8_attention_fits, a) : st;
}

}  // namespace

extern "C" {

size_t mg_kv8_code_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return cache_dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * 2 * 16 * head_dim : 0;
}

size_t mg_kv8_scale_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return cache_dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * 2 : 0;
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
