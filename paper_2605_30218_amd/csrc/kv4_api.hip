// kv4_api.hip -- the C entry points of the 4-bit paged K/V cache: host checks, then one launcher each.  See include/mg.h for the
// contract.
#include "mg_api_checks.h"

using namespace mg;

namespace {

// (a page of a head has a number of 31 bits: 2 TiB of codes)
bool dims_ok(int n_pages, int n_kv_heads, int head_dim) {
    return cache_dims_ok(n_pages, n_kv_heads, head_dim) && (int64_t)n_pages * n_kv_heads < (1ll << 31);
}
// MG_OK, or why the cache is refused
mg_status cache_status(const mg_kv4_cache* c) {
    if (!c || !c->codes || !c->scales || !aligned(c->codes, 16) || !aligned(c->scales, 4)) return MG_ERR_ARG;
    return dims_ok(c->n_pages, c->n_kv_heads, c->head_dim) ? MG_OK : MG_ERR_SHAPE;
}
Kv8 view(const mg_kv4_cache* c) { return Kv8{c->codes, c->scales, c->n_pages, c->n_kv_heads, c->head_dim}; }
// the checked arguments of an attention call as the kernels take them
mg_status attn_args(const mg_kv4_cache* c, const mg_kv8_attn_args* g, Kv8AttnArgs* a) {
    const mg_status st = cache_status(c);
    return st == MG_OK ? attn_args(view(c), g, kv4_attention_fits, a) : st;
}

constexpr int64_t MOST_PAIRS = 1 << 26;
// of an append: a token's values take 64 threads for each four KV heads, its heads at most 4 each, and a launch takes fewer than 2^32
constexpr int64_t MOST_TOKENS = 1 << 25;
static_assert(16 * (MOST_PAIRS + 3 * MOST_TOKENS) + 4 * (MOST_PAIRS + MOST_TOKENS) + 512 < 1ll << 32, "an append is one launch");

// n rows of `width` bf16 values
struct Rows {
    const uint16_t* p;
    int64_t stride, width;
    bool overlaps(const Rows& o, int64_t n) const {
        if (!n || !width || !o.width) return false;
        const int64_t a = reinterpret_cast<intptr_t>(p) / 2, b = reinterpret_cast<intptr_t>(o.p) / 2;
        if (a + (n - 1) * stride + width <= b || b + (n - 1) * o.stride + o.width <= a) return false;
        if (stride != o.stride) return true;
        // rows of the same stride may lie side by side, as the columns of one buffer
        const int64_t d = ((b - a) % stride + stride) % stride;
        return d < width || d + o.width > stride;
    }
};

}  // namespace

extern "C" {

size_t mg_kv4_code_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * 2 * 8 * head_dim : 0;
}

size_t mg_kv4_scale_bytes(int n_pages, int n_kv_heads, int head_dim) {
    return dims_ok(n_pages, n_kv_heads, head_dim) ? (size_t)n_pages * n_kv_heads * (head_dim / 2 + 16) : 0;
}

mg_status mg_kv4_append(const mg_kv4_cache* cache, const mg_kv4_append_args* g, void* stream) {
    const mg_status st = cache_status(cache);
    if (st != MG_OK) return st;
    if (!g || g->n_tokens < 0) return MG_ERR_ARG;
    if (g->n_q_heads < 0 || g->n_q_heads > 4096) return MG_ERR_SHAPE;
    if (g->n_tokens > MOST_TOKENS || (int64_t)g->n_tokens * (g->n_q_heads + cache->n_kv_heads) > MOST_PAIRS) return MG_ERR_ARG;
    if (g->n_tokens == 0) return MG_OK;
    const int64_t hd = cache->head_dim, kw = hd * cache->n_kv_heads, qw = hd * g->n_q_heads;
    if (!g->k || !g->v || !g->slots || !rows_ok(g->k, g->k_stride, kw) || !rows_ok(g->v, g->v_stride, kw)) return MG_ERR_ARG;
    if (g->positions && (!g->rope || !aligned(g->rope, 16) || g->n_positions < 1)) return MG_ERR_ARG;
    if (g->n_q_heads) {
        if (!g->q || !g->q_out || !rows_ok(g->q, g->q_stride, qw) || !rows_ok(g->q_out, g->q_out_stride, qw)) return MG_ERR_ARG;
        const Rows out{g->q_out, g->q_out_stride, qw};
        const bool same = g->q_out == g->q && g->q_out_stride == g->q_stride;
        if ((!same && out.overlaps(Rows{g->q, g->q_stride, qw}, g->n_tokens)) || out.overlaps(Rows{g->k, g->k_stride, kw}, g->n_tokens) ||
            out.overlaps(Rows{g->v, g->v_stride, kw}, g->n_tokens))
            return MG_ERR_ARG;
    }
    const Kv4AppendArgs a{view(cache), g->n_tokens, g->n_q_heads, g->q,      g->q_out,     g->k,    g->v,          g->q_stride,
                          g->q_out_stride, g->k_stride, g->v_stride, g->slots, g->positions, g->rope, g->n_positions};
    return status_of(launch_kv4_append(a, static_cast<hipStream_t>(stream)));
}

mg_status mg_kv4_read(const mg_kv4_cache* cache, int n, const int32_t* slots, uint16_t* k, int64_t k_stride, uint16_t* v,
                      int64_t v_stride, void* stream) {
    const mg_status st = cache_status(cache);
    if (st != MG_OK) return st;
    if (n < 0 || (int64_t)n * cache->n_kv_heads > MOST_PAIRS) return MG_ERR_ARG;
    if (n == 0 || (!k && !v)) return MG_OK;
    const int64_t w = (int64_t)cache->n_kv_heads * cache->head_dim;
    if (!slots || (k && !rows_ok(k, k_stride, w)) || (v && !rows_ok(v, v_stride, w))) return MG_ERR_ARG;
    return status_of(launch_kv4_read(view(cache), n, slots, k, k_stride, v, v_stride, static_cast<hipStream_t>(stream)));
}

size_t mg_kv4_attention_workspace_bytes(const mg_kv4_cache* cache, const mg_kv8_attn_args* args) {
    Kv8AttnArgs a{};
    if (attn_args(cache, args, &a) != MG_OK || a.T == 0 || a.B == 0) return 0;
    return kv4_attention_ws_bytes(a);
}

mg_status mg_kv4_attention(const mg_kv4_cache* cache, const mg_kv8_attn_args* args, void* workspace, size_t workspace_bytes,
                           void* stream) {
    Kv8AttnArgs a{};
    const mg_status st = attn_args(cache, args, &a);
    if (st != MG_OK) return st;
    if (a.T == 0 || a.B == 0) return MG_OK;
    if (a.out == a.q) return MG_ERR_ARG;
    const size_t need = kv4_attention_ws_bytes(a);
    if (need && (!workspace || workspace_bytes < need)) return MG_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return MG_ERR_ARG;
    a.part = static_cast<float*>(workspace);
    return status_of(launch_kv4_attention(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
