/*
 * mg.h -- C ABI of libmg.so, the MI355X (gfx950) hot path of MarginGate
 * (arXiv 2605.30218): one synchronous decode step of a batch of requests, the
 * top-1/top-2 margin gate, the deterministic verifier on the gated rows, and the
 * single-column K/V repair.
 *
 * Conventions for every call below
 *  - Pointers marked [device] are HIP device pointers owned by the caller; the
 *    library never frees them and keeps none of them beyond the call, except the
 *    weights, KV pool and workspace handed to mg_create, which must outlive the
 *    context.  Pointers marked [host] are read during the call only.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).  Every
 *    call only enqueues work on that stream and returns; results are ready when
 *    the stream is synchronised.  Kernel faults surface at that synchronisation.
 *  - Arguments the host can check (null pointers, sizes, batch above max_batch)
 *    return an error status and enqueue nothing.  Device-resident values (token
 *    ids, positions, page ids, row lists) are trusted: out-of-range values are
 *    the caller's error and are NOT checked on the device.
 *  - No call allocates device memory after mg_create.  One host thread at a time
 *    may use a given context; calls that overlap on different streams race on
 *    the context's workspace.
 *
 * Data layout
 *  - bf16 values are raw uint16 bit patterns.  Linear weights use the [out][in]
 *    row-major layout.  Logits are fp32.
 *  - Weight pointer table (mg_weight_count() entries, [device] bf16):
 *      [0] embed [V][d]
 *      layer l at 1 + 12*l: +0 attn_norm[d] +1 wq[Hq*hd][d] +2 wk[Hkv*hd][d]
 *        +3 wv[Hkv*hd][d] +4 bq[Hq*hd] +5 bk[Hkv*hd] +6 bv[Hkv*hd] (NULL when
 *        qkv_bias == 0) +7 wo[d][Hq*hd] +8 ffn_norm[d] +9 w_gate[F][d]
 *        +10 w_up[F][d] +11 w_down[d][F]
 *      [1 + 12*L] final_norm[d]   [2 + 12*L] lm_head[V][d]
 *  - KV pool: [layer][page][K|V][Hkv][page_size][hd] bf16.  K is stored after
 *    RoPE.  One head's page is page_size*hd contiguous values.
 *  - Page table: [B][max_pages_per_row] int32; position p of row b lives in page
 *    page_table[b*max_pages_per_row + p/page_size], slot p % page_size.  The
 *    caller allocates pages on the host; the page holding a row's current
 *    position must be mapped before the step.
 *  - A verifier K/V column of one row: [layer][K|V][Hkv][hd] bf16
 *    (mg_kv_col_elems() values).
 */
#ifndef MG_H
#define MG_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MG_OK = 0,
    MG_ERR_ARG = -1,       /* null pointer or value out of range */
    MG_ERR_SHAPE = -2,     /* model shape the kernels do not support */
    MG_ERR_WORKSPACE = -3, /* workspace or KV pool smaller than required */
    MG_ERR_HIP = -4,       /* a HIP runtime call failed */
    MG_ERR_STATE = -5      /* call not valid in the context's current state */
} mg_status;

typedef struct {
    int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab;
    int32_t qkv_bias;          /* 1: q/k/v projections carry a bias */
    float rope_theta, rms_eps;
    int32_t page_size;         /* must be 16 */
    int32_t max_batch;         /* rows per step, 1..256 */
    int32_t max_pages_per_row; /* page-table row stride; max position = this * page_size - 1 */
    int32_t n_pages;           /* pages in the KV pool */
    int32_t max_prefill;       /* items per mg_prefill call (0 = 1024) */
} mg_model_cfg;

typedef struct mg_ctx mg_ctx;

/* Entries of the weight pointer table: 3 + 12 * n_layers. */
int mg_weight_count(const mg_model_cfg* cfg);
/* Bytes of the KV pool the shape needs: n_layers*n_pages*2*Hkv*page_size*hd*2. */
size_t mg_kv_pool_bytes(const mg_model_cfg* cfg);
/* bf16 values of one row's K/V column: n_layers*2*Hkv*hd. */
size_t mg_kv_col_elems(const mg_model_cfg* cfg);
/* Bytes of device workspace mg_create needs (0 if the shape is unsupported). */
size_t mg_workspace_bytes(const mg_model_cfg* cfg);
const char* mg_status_string(int status);

/* Create a context.  Checks the shape (d_model, d_ffn, Hq*hd multiples of 64;
 * head_dim 64 or 128; Hq % Hkv == 0; page_size 16), copies the RoPE table into
 * the workspace and zeroes the workspace's counters (synchronous).  weights
 * [host array of device pointers], kv_pool and workspace [device]. */
mg_status mg_create(const mg_model_cfg* cfg, const void* const* weights, void* kv_pool, size_t kv_pool_bytes,
                    void* workspace, size_t workspace_bytes, mg_ctx** out);
mg_status mg_destroy(mg_ctx* ctx);

/* (1) The BF16 fast path: the ordinary batched decoder forward whose logits the
 * gate inspects (paper Sec. 3.1, margin trigger), which also writes the current
 * token's K/V column into the cache as a tentative entry (Sec. 3.2).  For each row b < B: consumes tokens[b] at position
 * positions[b], writes that position's K (after RoPE) and V into the paged
 * cache in every layer, attends over positions 0..positions[b], and writes
 * fp32 logits[b][V].  Its reduction plan depends on B (it may differ in the last
 * bits between batch sizes; that is the effect the method guards against).
 * tokens, positions [device int32, B]; page_table [device int32,
 * B*max_pages_per_row]; logits [device fp32, B*V]. */
mg_status mg_decode_step(mg_ctx* ctx, int B, const int32_t* tokens, const int32_t* positions,
                         const int32_t* page_table, float* logits, void* stream);

/* (2) The margin gate (Sec. 3.1): per row, top1[b] = argmax (lowest index on
 * ties), margin[b] = l_(1) - l_(2) where l_(2) is the second largest value of
 * the row (0 when the maximum is duplicated; NaN when the row holds a NaN),
 * gate[b] = protected[b] && !(margin[b] >= tau), i.e. the strict trigger
 * g < tau with NaN firing.  gated_rows receives the gated row indices in
 * increasing order and *n_gated their count (device scalar), so the verifier can
 * be launched on exactly those rows (the repair request of Sec. 3.2).
 * logits [device fp32 B*V]; protected_mask [device uint8 B] or NULL (= all rows
 * protected, Sec. 3.3's per-request policy); top1, gated_rows [device int32 B];
 * margin [device fp32 B]; gate [device uint8 B]; n_gated [device int32 1].
 * n_gated_host: NULL, or one int32 of pinned host memory (allocated with
 * hipHostMalloc) that also receives the count, stored with system scope after
 * gated_rows and *n_gated are written, so a host can poll it instead of
 * synchronising the stream (the caller sets it to a negative value first).
 * Bit-exact: comparisons only, no rounding. */
mg_status mg_margin_gate(mg_ctx* ctx, int B, const float* logits, const uint8_t* protected_mask, float tau,
                         int32_t* top1, float* margin, uint8_t* gate, int32_t* gated_rows, int32_t* n_gated,
                         int32_t* n_gated_host, void* stream);

/* The margin gate of mg_margin_gate for callers that cannot allocate device memory or hold
 * a context: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same outputs and the same bits as mg_margin_gate over B rows of V logits
 * (B <= 256, V >= 2, else MG_ERR_ARG), without the host-mirror count.  Its partial states
 * live in a static device array of 33 KiB per GPU, held until the process ends; the first
 * call on a device looks up that array's address (no allocation, no context).  Every call
 * on one GPU shares that array: calls that overlap on one GPU (different streams, or
 * different host threads) race and must be serialised by the caller.  All pointers
 * [device], as in mg_margin_gate; stream as everywhere. */
mg_status mg_margin_gate_noalloc(int B, int V, const float* logits, const uint8_t* protected_mask, float tau,
                                 int32_t* top1, float* margin, uint8_t* gate, int32_t* gated_rows, int32_t* n_gated,
                                 void* stream);

/* (3) The deterministic verifier (Sec. 3.2, deterministic verifier contract):
 * runs the current step again for rows rows[0..n) of the step batch with
 * the canonical reduction order (fixed per-lane groups + xor butterfly for dot
 * products, chunks of 256 positions for attention, own EXP), which depends on
 * neither n, nor the row's place in the list, nor the batch.  The row attends
 * over cache positions 0..positions[r]-1 as committed plus its OWN current
 * column, never the tentative one.  Outputs for list entry i: v_logits[i][V]
 * (fp32, may be NULL), v_tok[i] = argmax (lowest index on ties), and the K/V
 * column v_kvcol[i] (bf16, mg_kv_col_elems values).  The cache is not written.
 * n >= 0: host count.  n == -1: the count is read on the device from *n_dev
 * (graph-capturable), bounded by max_batch.  rows [device int32 n]; tokens,
 * positions, page_table as in mg_decode_step. */
mg_status mg_verify_rows(mg_ctx* ctx, int n, const int32_t* rows, const int32_t* n_dev, const int32_t* tokens,
                         const int32_t* positions, const int32_t* page_table, float* v_logits, int32_t* v_tok,
                         uint16_t* v_kvcol, void* stream);

/* A matrix-core verifier for the n listed rows (host count): the BF16 forward on
 * v_mfma_f32_16x16x32_bf16 (the fast path's kernels) with every projection's split-K
 * fixed as for 32 rows, so a row's arithmetic depends on neither n nor its place in the
 * list -- deterministic and batch-invariant by fixed tiling, which is what the
 * deterministic verifier contract of Sec. 3.2 asks for.  Its order is not the canonical
 * one of mg_verify_rows: its results match the oracle within the fast path's tolerance,
 * not bit for bit.  Outputs as mg_verify_rows: v_logits [n][vocab] fp32 (may be NULL: then
 * the LM head runs with a fused top-2 epilogue that writes no logits, and v_tok is the same
 * index), v_tok[i] = argmax (lowest index on ties), v_kvcol[i] the row's K/V column [L][2][Hkv][hd]
 * bf16; the cache is read (positions < positions[rows[i]]) and not written.  Shares the
 * context's workspace with the other calls (one call at a time per context). */
mg_status mg_verify_rows_mfma(mg_ctx* ctx, int n, const int32_t* rows, const int32_t* tokens,
                              const int32_t* positions, const int32_t* page_table, float* v_logits, int32_t* v_tok,
                              uint16_t* v_kvcol, void* stream);

/* (4) Commit and single-column repair (Sec. 3.2): for list entry i with row
 * r = rows[i]: emitted[r] = v_tok[i]; if v_tok[i] != top1[r] the verifier's
 * column v_kvcol[i] overwrites the cache at position positions[r] in every
 * layer and *n_repaired is incremented (device int32, accumulates over calls).
 * When the tokens agree the tentative column stays (verified commit).  Rows not
 * listed keep emitted[r] as the caller set it (normally top1[r]); emitted may be
 * the same buffer as top1.  n / n_dev as in mg_verify_rows. */
mg_status mg_repair_kv_column(mg_ctx* ctx, int n, const int32_t* rows, const int32_t* n_dev,
                              const int32_t* positions, const int32_t* page_table, const int32_t* top1,
                              const int32_t* v_tok, const uint16_t* v_kvcol, int32_t* emitted,
                              int32_t* n_repaired, void* stream);

/* The same commit with a choice of repair action (the variants around the rule of
 * Sec. 3.2; Sec. 4, Ablations and Robustness, describes the token-only one):
 *   MG_REPAIR_ON_MISMATCH  the method: copy the verifier column when v_tok[i] != top1[r]
 *                          (mg_repair_kv_column is this action);
 *   MG_REPAIR_TOKEN_ONLY   emit the verifier token, never copy (the tentative BF16 column
 *                          stays; *n_repaired is not incremented);
 *   MG_REPAIR_COPY_ALWAYS  copy the verifier column for every listed row, agreeing rows
 *                          included (*n_repaired counts every copy).
 * Arguments, layout and errors as mg_repair_kv_column; an action outside the three
 * returns MG_ERR_ARG and enqueues nothing. */
enum { MG_REPAIR_ON_MISMATCH = 0, MG_REPAIR_TOKEN_ONLY = 1, MG_REPAIR_COPY_ALWAYS = 2 };
mg_status mg_repair_kv_column_action(mg_ctx* ctx, int n, const int32_t* rows, const int32_t* n_dev,
                                     const int32_t* positions, const int32_t* page_table, const int32_t* top1,
                                     const int32_t* v_tok, const uint16_t* v_kvcol, int32_t* emitted,
                                     int32_t* n_repaired, int action, void* stream);

/* Prompt prefill with the verifier's canonical arithmetic, so that runs at any
 * batch size start from bit-identical prompt caches.  Item i consumes
 * tokens[i] at position positions[i] of row item_rows[i] (a row of page_table)
 * and writes that position's K/V into the cache.  Attention of an item reads
 * positions 0..positions[i] of its row, so every earlier position must be in
 * this call or an earlier one.  Items per call: at most max_prefill.  The result
 * for an item is bit-identical to a verifier recomputation at that position. */
mg_status mg_prefill(mg_ctx* ctx, int n_items, const int32_t* tokens, const int32_t* positions,
                     const int32_t* item_rows, const int32_t* page_table, void* stream);

/* Step bookkeeping: tokens[b] = emitted[b]; positions[b] += 1 for b < B. */
mg_status mg_advance(mg_ctx* ctx, int B, const int32_t* emitted, int32_t* tokens, int32_t* positions,
                     void* stream);

/* ---- (5) batch planning and an 8-bit paged K/V cache -------------------------------------
 *
 * For serving programs whose decode is bound by the bytes of the K/V cache: the cache of a
 * layer at one byte a value, with the append that quantises into it, the attention that reads
 * it, and the plan of a batch's pages and slots.  None of these calls needs a context; they
 * keep no state, allocate nothing, and can be captured into a HIP graph (a replay reads the
 * lengths, tables and slots that the device buffers then hold).  Calls on different streams may
 * run at once where they write different buffers (pages, workspaces and outputs).
 *
 * A page holds 16 positions.  Slot = page * 16 + position % 16.  The cache of one layer:
 *   codes  [n_pages][Hkv][K|V][16 * hd]  e4m3 values (OCP: 4 exponent bits, 3 mantissa bits,
 *          largest 448, no infinity, 0x7f / 0xff NaN)
 *   scales [n_pages][Hkv][K|V]           b; a code stands for its value * 2^(b - 127).  0: nothing stored, else
 *          16..254 (mg_kv8_append needs no more than 247 of its own; a page that another program filled may have more)
 * so one scale serves 16 positions of one KV head.  Order inside a page of a head, chosen so
 * that a wave reads matrix operands as contiguous 1 KiB runs:
 *   K: position t, feature d = 64 h + 16 g + j at byte ((h * 4 + g) * 16 + t) * 16 + j
 *   V: position t = 4 g + i, feature d = 64 h + 16 c + m at byte ((h * 4 + g) * 16 + m) * 16 + 4 c + i
 * A value read back is exact in bf16 (but for codes that stand for 2^128 or more, infinity: finite values
 * above 1.9375 * 2^127 round to 2^128).  A zeroed pool is an empty cache. */
typedef struct {
    uint8_t* codes;   /* [device], 16-byte aligned */
    uint8_t* scales;  /* [device], 2-byte aligned */
    int32_t n_pages;  /* 1..2^27 - 1 */
    int32_t n_kv_heads;
    int32_t head_dim; /* 64 or 128 */
} mg_kv8_cache;

/* Bytes of the two buffers of one layer (0 if the shape is unsupported). */
size_t mg_kv8_code_bytes(int n_pages, int n_kv_heads, int head_dim);
size_t mg_kv8_scale_bytes(int n_pages, int n_kv_heads, int head_dim);

/* Pages, slots and per-token lists of a batch from its requests' lengths, in one launch.
 * Row b holds ctx_len[b] positions and asks for n_new[b] more.  It is valid when both are >= 0
 * and their sum fits its page-table row (16 * max_pages_per_row positions).  Rows are admitted
 * in order: a valid row is admitted when the new pages of all valid rows up to and including it
 * are at most *n_free and their new tokens at most max_tokens (the first that does not fit stops
 * the rows behind it; an invalid row stops nobody).  Every admitted row gets pages for positions
 * ctx_len[b] .. ctx_len[b] + n_new[b] - 1: those it lacks are taken from the end of
 * free_pages[0 .. *n_free) in row order and written to its entries of page_table; all other
 * entries are left as they were.
 *   cu_new [B + 1]: tokens of the admitted rows before row b;  lens [B]: positions after the call
 *   (ctx_len[b] where not admitted, 0 where that is negative);  admitted [B] 0 or 1;
 *   positions, rows, slots [max_tokens]: of every new token, row by row, positions ascending
 *   (the item lists of mg_prefill; the slots of mg_kv8_append), -1 behind the last; also the slot of a
 *   token whose page-table entry is no page (outside 0 .. 2^27 - 1);
 *   *n_left: free pages that remain, so that free_pages[0 .. *n_left) is the next call's list.
 * free_pages must be distinct pages that no row holds.  1 <= B <= 1024.  All pointers [device];
 * no output may overlap an input or the page table, nor that an input (blocks of the launch read
 * one while others write): MG_ERR_ARG. */
mg_status mg_batch_plan(int B, int max_pages_per_row, const int32_t* ctx_len, const int32_t* n_new,
                        const int32_t* free_pages, const int32_t* n_free, int max_tokens, int32_t* page_table,
                        int32_t* cu_new, int32_t* lens, int32_t* admitted, int32_t* positions, int32_t* rows,
                        int32_t* slots, int32_t* n_left, void* stream);

/* Quantises the K (after RoPE) and V rows of n_tokens tokens into the cache.  Token t's row is
 * k + t * k_stride values (bf16 [Hkv][hd]; likewise v) and goes to slots[t]; a slot outside the
 * cache (the plan's -1) is skipped.  Tokens of one page must stand together, in ascending slots
 * without gaps (as the plan lists them): of a page that two separate runs of one call write, the same
 * slot twice among them, the content is undefined (of no other page).  For a page and head, with need = the least b in [16, 254] with
 * amax <= 448 * 2^(b - 127) over the finite values that the call writes there:
 *   - a run that begins at the page's position 0, or a page whose scale is 0, starts anew: scale =
 *     need, the page's other positions become 0;
 *   - else scale = max(old scale, need); when it grows the page's other positions are rounded
 *     once more, to the new scale.
 * A code is the nearest e4m3 value, ties to even; a value that is not finite becomes NaN.  The
 * outcome depends neither on the split of a page's tokens over calls nor on the launch, except
 * where a value falls below its scale's normal range (2^-6) and is rounded again as it grows.
 * k, v 16-byte aligned [device], strides multiples of 8 and >= Hkv * hd; at most 2^26 (token, KV
 * head) pairs a call. */
mg_status mg_kv8_append(const mg_kv8_cache* cache, int n_tokens, const uint16_t* k, int64_t k_stride,
                        const uint16_t* v, int64_t v_stride, const int32_t* slots, void* stream);

/* The values of n slots as bf16 rows (exact): slot slots[i]'s K [Hkv][hd] at k + i * k_stride and V
 * likewise; either of k, v may be NULL.  Rows of slots outside the cache are left as they were.
 * For handing a request's cache to another program (a context's bf16 pool keeps a page's positions head by
 * head, so the caller places these rows there itself).  Alignment and strides as in mg_kv8_append. */
mg_status mg_kv8_read(const mg_kv8_cache* cache, int n, const int32_t* slots, uint16_t* k, int64_t k_stride,
                      uint16_t* v, int64_t v_stride, void* stream);

/* Attention of a batch's new tokens over the cache.  Row b has the tokens cu_new[b] ..
 * cu_new[b + 1] - 1 of q (cu_new NULL: token b alone), the last of them at position lens[b] - 1, so
 * its token i of n stands at p = lens[b] - n + i; their own K/V are in the cache already.  A token sees
 * the positions j <= p, j > p - window (window > 0), whose page-table entry is a page of the cache
 * (entries outside 0 .. n_pages - 1 are holes, and so is what a length past the table lacks).  With s_j = scale * q . k_j, or softcap *
 * tanh(scale * q . k_j / softcap) where softcap > 0: out = sum_j softmax(s)_j v_j, rounded once to bf16; a
 * token that sees nothing gets zeros.  What stands at a position that a token does not see has no effect on
 * it, NaN and infinity among it; a value of V that reads as NaN or infinity makes its feature NaN or infinity
 * in the tokens that see it.  Query head h reads KV head h / (Hq / Hkv).  Rows without tokens and rows of out behind
 * the last token are left as they were.
 * Scores are fp32 numbers; they have to stay within 2^23 of zero (the exponents' reference is rounded with them: from some 2^30 on a row's
 * outputs become NaN or zeros).  Sums are fp32 of terms up to 2^9 above their weights on average, so features overflow where |v| passes some
 * 2^116 / (positions seen); a probability enters the product with V as two bf16 terms (16 bits) where a row has
 * few query rows (tokens times query heads of a KV head: up to 16, or 32 where no row of the call has
 * more), and as one (8 bits, as an output's) in longer chunks.  The order of a row's sums follows the
 * call's shape (rows, tokens, bounds) and the lengths, so the same call gives the same bits.  Calls whose
 * launch would pass 2^22 blocks (some millions of rows, or of tokens) are refused: MG_ERR_ARG. */
typedef struct {
    int32_t n_rows, n_tokens;
    int32_t n_q_heads;         /* a multiple of n_kv_heads, at most 16 times it */
    int32_t max_new;           /* at least the most tokens of any row (a row with more is the caller's error) */
    int32_t max_len;           /* host bound on lens, for the launch's shape only (0: the page table's capacity) */
    int32_t max_pages_per_row; /* page-table row stride, 1..2^26 */
    int32_t window;            /* 0: every earlier position */
    float scale;               /* 0: 1 / sqrt(head_dim); else 1e-15 .. 1e15 */
    float softcap;             /* 0: none; else 1e-15 .. 1e15 */
    const uint16_t* q;         /* [device] bf16 [n_tokens][Hq][hd], token stride q_stride values */
    int64_t q_stride;
    uint16_t* out;             /* [device] as q, token stride out_stride; must not overlap q (equal: MG_ERR_ARG) */
    int64_t out_stride;
    const int32_t* page_table; /* [device] [n_rows][max_pages_per_row] */
    const int32_t* lens;       /* [device] [n_rows] */
    const int32_t* cu_new;     /* [device] [n_rows + 1], or NULL */
} mg_kv8_attn_args;
/* Bytes of workspace the call needs on the current device (host logic; 0 also where the arguments
 * are refused).  The workspace holds nothing between calls. */
size_t mg_kv8_attention_workspace_bytes(const mg_kv8_cache* cache, const mg_kv8_attn_args* args);
mg_status mg_kv8_attention(const mg_kv8_cache* cache, const mg_kv8_attn_args* args, void* workspace,
                           size_t workspace_bytes, void* stream);

/* ---- (6) a 4-bit paged K/V cache, with the rotation of positions ------------------------------
 *
 * As (5), at half a byte a value: pages of 16 positions, slots and plans are the same, and so is what is said there of
 * contexts, allocations, graphs and streams.  The cache of one layer, in the microscaling format of 4 bits:
 *   codes  [n_pages][Hkv][K|V][8 * hd]  two e2m1 values a byte, the low nibble first (0, 0.5, 1, 1.5, 2, 3, 4, 6, bit 3 the sign)
 *   scales [n_pages][Hkv][hd / 2 + 16]  b; a code stands for its value * 2^(b - 127).  255: the block holds a value that is not
 *          finite, and all of it reads as NaN; else 16..253 where mg_kv4_append wrote it, 0 where nothing is stored
 * A block is 32 features of a position's key, or a position's whole value of a KV head; its scale is the least power of two whose
 * sevenfold holds its largest magnitude (what lies between 6 and 7 times it becomes 6).  Codes are the nearest, ties to even.
 * So a position's codes depend on its own row alone, and nothing is rounded twice.  Order inside a page of a head:
 *   K: position t, feature d = 32 g + j at byte (g * 16 + t) * 16 + j / 2, nibble j % 2; scale byte g * 16 + t
 *   V: position t = 4 g + i, feature d = 16 c + m at byte (g * 16 + m) * hd / 8 + 2 c + i / 2, nibble i % 2; scale byte hd / 2 + t
 * which is the order of the matrix instructions' 4-bit operands.  A value read back is exact in bf16 (but for codes that stand for
 * 2^128 or more, infinity: finite values from 1.75 * 2^127 may become such a one).  A zeroed pool is an empty cache. */
typedef struct {
    uint8_t* codes;   /* [device], 16-byte aligned */
    uint8_t* scales;  /* [device], 4-byte aligned */
    int32_t n_pages;  /* 1..2^27 - 1, n_pages * n_kv_heads < 2^31 */
    int32_t n_kv_heads;
    int32_t head_dim; /* 64 or 128 */
} mg_kv4_cache;

/* Bytes of the two buffers of one layer (0 if the shape is unsupported). */
size_t mg_kv4_code_bytes(int n_pages, int n_kv_heads, int head_dim);
size_t mg_kv4_scale_bytes(int n_pages, int n_kv_heads, int head_dim);

/* The new tokens' rows of a QKV projection into the cache, rotated on the way: for token i with position p = positions[i], every
 * query head of q (n_q_heads of them; 0: none, q and q_out are not read) is rotated and written to q_out, every key of k is rotated
 * and stored at slots[i], and v is stored there as it is.  Rotating a head x by p: with c, s = rope[p][2 j], rope[p][2 j + 1],
 *   x'[j] = x[j] c - x[j + hd / 2] s,  x'[j + hd / 2] = x[j + hd / 2] c + x[j] s,   j < hd / 2,
 * products and sums each rounded to fp32, x' to bf16 (the table and the arithmetic of mg_decode_step).  positions NULL: nothing is
 * rotated (rope is not read; q is copied to q_out).
 * Tokens with a negative position are left out: nothing is written for them.  A slot outside the cache stores nothing (its q is
 * rotated).  A position of n_positions or more has no angle: its q_out and key become NaN.
 * Tokens may stand in any order (the plan's, where neighbouring positions are neighbours, is the fastest), and positions that the call has no token for are
 * left as they were.  Two tokens with the same slot leave its key undefined; its value is the later one's where they stand within four consecutive
 * tokens, else the values of its four aligned positions (4 g .. 4 g + 3 of a page) are undefined.
 * q, k, v, q_out bf16 [n][heads][hd], 16-byte aligned, strides in values, multiples of 8 and >= heads * hd.  q_out may be q
 * itself (with q's stride); else no written row may overlap a row of q, k or v: MG_ERR_ARG.  At most 2^25 tokens and
 * 2^26 (token, head) pairs of q and k a call.  slots, positions int32 [n]; rope fp32 [n_positions][hd], 16-byte aligned. */
typedef struct {
    int32_t n_tokens;
    int32_t n_q_heads;         /* 0..4096 */
    const uint16_t* q;
    int64_t q_stride;
    uint16_t* q_out;
    int64_t q_out_stride;
    const uint16_t* k;
    int64_t k_stride;
    const uint16_t* v;
    int64_t v_stride;
    const int32_t* slots;
    const int32_t* positions;  /* or NULL */
    const float* rope;         /* with positions */
    int32_t n_positions;       /* rows of rope */
} mg_kv4_append_args;
mg_status mg_kv4_append(const mg_kv4_cache* cache, const mg_kv4_append_args* args, void* stream);

/* As mg_kv8_read: the values of n slots as bf16 rows. */
mg_status mg_kv4_read(const mg_kv4_cache* cache, int n, const int32_t* slots, uint16_t* k, int64_t k_stride,
                      uint16_t* v, int64_t v_stride, void* stream);

/* As mg_kv8_attention, over this cache: the same arguments, visibility, order and refusals.
 * A value of K or V that is NaN (a scale byte of 255) makes the outputs of the tokens that see it NaN, of V in all features; so do a
 * query value that is not finite and sums past fp32, which are reached where |v| passes some 2^100.  Query values enter as three 6-bit terms
 * under the scale of 32 features: exact but for those below 2^-6 of their block's largest, which are off by at most 2^-14 of that.
 * A probability times its value's scale enters the product with V as two such terms, or more where 32 positions' scales are more than 2^2 apart: a
 * probability is off by at most 2^-8 of itself or 1/480 of the largest of 32 positions, whichever is more, whatever the sizes of their values (and by some
 * 2^-116 over its value's scale: where all |v| of a row are below some 2^-100 its outputs lose bits).  Scores may be any fp32 numbers. */
size_t mg_kv4_attention_workspace_bytes(const mg_kv4_cache* cache, const mg_kv8_attn_args* args);
mg_status mg_kv4_attention(const mg_kv4_cache* cache, const mg_kv8_attn_args* args, void* workspace,
                           size_t workspace_bytes, void* stream);

/* ---- (7) log probabilities of tokens ---------------------------------------------------------
 *
 * For answers and scores with log probabilities, from the logits that the margin gate reads: for each row r of n, with
 * lse = ln sum_j e^logits[r][j],
 *   logprob[r] = logits[r][tokens[r]] - lse (NaN where tokens[r] is outside 0..vocab - 1),
 *   entropy[r] = - sum_j p_j ln p_j,  p_j = e^(logits[r][j] - lse),
 *   top_tokens[r][i], top_logprobs[r][i], i < top: the row's largest logits in falling order, the lower index first among equal
 *   ones, and their log probabilities; -1 and -inf where fewer than `top` logits are above -inf.
 * Logits of -inf are masked: they have no part in the sums.  A row that is masked whole has log probabilities of -inf and an
 * entropy of 0.  A NaN or +inf in a row makes its log probabilities and entropy NaN; NaN is never among the top tokens.
 * logits fp32 (logits_bf16 = 0) or bf16, row stride `stride` values (>= vocab, any alignment of a value); 1 <= vocab <= 2^30,
 * 0 <= top <= 32, top <= vocab, n < 2^24.  logprob, entropy [n], top_tokens, top_logprobs [n][top]: any may be NULL (with
 * logprob NULL tokens are not read).  No output may overlap the logits or tokens.  The workspace holds nothing between calls; the
 * same call gives the same bits. */
size_t mg_token_logprobs_workspace_bytes(int n, int vocab, int top);
mg_status mg_token_logprobs(int n, int vocab, const void* logits, int logits_bf16, int64_t stride, const int32_t* tokens,
                            int top, float* logprob, float* entropy, int32_t* top_tokens, float* top_logprobs,
                            void* workspace, size_t workspace_bytes, void* stream);

/* ---- measurement hooks (used by the benchmark; not part of the method) ---- */

enum {
    MG_KIND_FAST_GEMM = 0,  /* weight-streaming projections of the fast path */
    MG_KIND_FAST_ATTN = 1,  /* paged decode attention of the fast path */
    MG_KIND_CANON_GEMV = 2, /* weight-streaming projections of the verifier */
    MG_KIND_CANON_ATTN = 3, /* paged decode attention of the verifier */
    MG_KIND_GATE = 4,       /* margin gate */
    MG_KIND_COUNT = 5
};

/* Start recording a HIP event pair around every launch of kernel class `kind`
 * (on the stream it is launched on), up to max_launches launches.  Creates the
 * events (not allocation-free; call outside timed loops).  The events are
 * timing-only: recording them performs no system-scope fence. */
mg_status mg_profile_begin(mg_ctx* ctx, int kind, int max_launches);
/* Stop recording, synchronise the device and report the number of
 * launches, their summed duration in milliseconds, the summed algorithmic bytes
 * (every weight, activation, K/V and output byte the launch must move once) and
 * the summed algorithmic flops (2 per multiply-add). */
mg_status mg_profile_end(mg_ctx* ctx, int kind, int* n_launches, double* total_ms, double* algo_bytes,
                         double* algo_flops);

#ifdef __cplusplus
}
#endif
#endif
