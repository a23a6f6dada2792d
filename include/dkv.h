/*
 * dkv.h - C boundary of the MI355X (gfx950) library for the delayed KV-cache (dKV-Cache) hot path
 * of masked diffusion language models (arxiv 2505.15781).
 *
 * The hot path is one denoising step: choose the rows to recompute, run the transformer on those
 * rows only, overwrite their K/V in a position-indexed cache, attend (unmasked) over all positions,
 * take the vocabulary softmax of the candidate rows and commit the most confident ones.
 *
 * Conventions
 *  - Every pointer is marked (dev) = device memory or (host) = host memory.
 *  - All device memory is owned by the caller (weights, cache, token state, logs, workspace) and
 *    must outlive the context. The library allocates only the small host-side context, and never
 *    device memory.
 *  - All device work is enqueued on the caller's HIP stream (a hipStream_t passed as void*); calls
 *    return without waiting for it, except the dkv_read_* debug calls and dkv_profile_end, which
 *    synchronise that stream.
 *  - Every call returns 0 on success or a negative DKV_E_* code; dkv_last_error() gives the text
 *    of the most recent failure on this thread. No call aborts or throws.
 *  - Positions are 0-based; the generated region is [prompt_len, prompt_len + gen_len).
 */
#ifndef DKV_H
#define DKV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* storage / arithmetic type of weights, activations fed to the projections, and the K/V cache;
 * accumulation, softmax, the residual stream and confidences are always fp32 */
#define DKV_BF16 0
#define DKV_FP32 1
#define DKV_E4M3 2        /* paged caches only (dkv_paged_cache): 8 bits per element, a scale per position and K/V head */
#define DKV_E2M1 4        /* paged caches only: 4 bits per element, a scale for each 32 dims of a position and K/V head */

/* cache variants (Sec. 3.3 "dKV-Cache-Decode", "dKV-Cache-Prefill and dKV-Cache-PD"; Sec. 3.4) */
#define DKV_DECODE  0
#define DKV_GREEDY  1
#define DKV_PREFILL 2
#define DKV_PD      3

/* remasking (Sec. 3.1 "Sampling Process"): keep the most confident, or a predefined order */
#define DKV_CONFIDENCE   0
#define DKV_RANDOM_ORDER 1

/* centre of the Greedy local window (Sec. 3.4): the position decoded now, or one step ago */
#define DKV_CENTER_CUR  0
#define DKV_CENTER_PREV 1

/* scope of an explicit refresh */
#define DKV_SCOPE_ALL 0
#define DKV_SCOPE_GEN 1

#define DKV_OK                     0
#define DKV_E_INVALID_ARG         -1
#define DKV_E_BAD_STATE           -2
#define DKV_E_UNSUPPORTED         -3
#define DKV_E_WORKSPACE_TOO_SMALL -4
#define DKV_E_HIP                 -5

typedef struct dkv_ctx dkv_ctx;

/* Pre-norm transformer block without biases: RMSNorm, rotary embedding (half-split pairing
 * i <-> i + head_dim/2), bidirectional attention with n_q_heads / n_kv_heads query heads sharing
 * each K/V head, SwiGLU feed-forward. head_dim must be 32, 64 or 128 and even. */
typedef struct {
    int32_t n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab, mask_id;
    int32_t dtype;                     /* DKV_BF16 or DKV_FP32 */
    float rms_eps, rope_theta;
} dkv_model_desc;

/* Weights, all (dev), row-major [out_features, in_features] so that y = x * W^T, elements of
 * model dtype; norm gains are fp32 in both modes.
 *   embed, lm_head [vocab, d_model]; final_norm [d_model]
 *   wqkv[l]      [(n_q_heads + 2 n_kv_heads) * head_dim, d_model]: Q rows (head-major), K rows, V rows
 *   wo[l]        [d_model, n_q_heads * head_dim]
 *   w_gate_up[l] [2 * d_ffn, d_model]: row 2j is gate_j, row 2j+1 is up_j
 *   w_down[l]    [d_model, d_ffn]
 *   norm1[l], norm2[l] [d_model]
 * The six per-layer members are (host) arrays of n_layers (dev) pointers; the arrays themselves
 * are copied during dkv_init_cache and need not outlive it. */
typedef struct {
    const void *embed, *lm_head;
    const float *final_norm;
    const void *const *wqkv, *const *wo, *const *w_gate_up, *const *w_down;
    const float *const *norm1, *const *norm2;
} dkv_weights;

/* The run: sequence, step schedule, refresh interval and variant.
 * Requirements (else DKV_E_INVALID_ARG): gen_len % block_len == 0; steps % (gen_len / block_len)
 * == 0; block_len % steps_per_block == 0 (k = block_len / steps_per_block positions are
 * committed per step per sequence); refresh_interval >= 1. Step 0 always recomputes everything;
 * afterwards step t is a scheduled refresh iff t % refresh_interval == 0 (Sec. 3.3, "Cache
 * Refreshing Mechanism"). */
typedef struct {
    int32_t batch, prompt_len, gen_len, steps, block_len, refresh_interval;
    int32_t variant;                   /* DKV_DECODE | DKV_GREEDY | DKV_PREFILL | DKV_PD */
    int32_t delay;                     /* 1: recompute the previous step's commits once more before
                                          caching them (Eq. 4); 0: cache at once (Eq. 3) */
    int32_t window, window_center, include_prev;   /* Greedy: window size w, its centre, and whether
                                                      the previous step's commits are recomputed */
    int32_t remask;                    /* DKV_CONFIDENCE | DKV_RANDOM_ORDER */
    int32_t shift_logits;              /* 0: the output at position q is the distribution of token q;
                                          1: of token q + 1 (models adapted from autoregressive ones,
                                          Appendix B, K/V cached unshifted): the row before every
                                          position that may be committed joins the active set and
                                          supplies its logits. Needs prompt_len >= 1. */
    const int32_t *order;              /* (dev) [batch, gen_len] absolute positions in commit order;
                                          DKV_RANDOM_ORDER only (required by DKV_GREEDY) */
} dkv_run_desc;

/* Caller-owned device state. k_cache / v_cache hold post-rotation keys and values of every
 * position: [n_layers][batch][n_kv_heads][seq_len][head_dim], model dtype, seq_len = prompt_len +
 * gen_len. tokens must hold the prompt ids in [:, :prompt_len] before dkv_init_cache.
 * decoded_* are logs of what each step committed, [steps][batch][k]. */
typedef struct {
    void *k_cache, *v_cache;           /* (dev) */
    int32_t *tokens;                   /* (dev) [batch, seq_len], in/out */
    uint8_t *masked;                   /* (dev) [batch, seq_len], 1 = not yet finalised */
    int32_t *stamp;                    /* (dev) [batch, seq_len], last step that wrote K/V; -1 never */
    int32_t *decoded_pos, *decoded_tok;/* (dev) [steps, batch, k] */
    float *decoded_conf;               /* (dev) [steps, batch, k] */
    void *workspace;                   /* (dev) scratch, 256-byte aligned */
    size_t workspace_bytes;
} dkv_buffers;

/* Bytes of workspace dkv_init_cache needs for this model and run (0 on invalid descriptors). */
size_t dkv_workspace_bytes(const dkv_model_desc *model, const dkv_run_desc *run);

/* Bind buffers and start a run: generated region of tokens := mask_id, masked := [p >= prompt_len],
 * stamp := -1, logs cleared, step counter := 0 (state before the first step of Sec. 3.1's sampling
 * process). The descriptors are copied. `stream` is a hipStream_t. */
int dkv_init_cache(dkv_ctx **out, const dkv_model_desc *model, const dkv_weights *weights,
                   const dkv_run_desc *run, const dkv_buffers *buffers, void *stream);

/* Compute the active set A_t of step `step` on the device (Eq. 4: everything still masked plus the
 * previous step's commits; all positions, or the generated region, on a refresh; the Greedy set
 * of Sec. 3.4). Rows are ordered sequence by sequence, position ascending.
 * active_idx (dev, nullable) receives the positions and must have room for batch * seq_len entries:
 * the call copies as many entries as the schedule's bound below says, which is not known before the
 * call and can exceed the true row count; entries from active_off[batch] on are undefined.
 * active_off (dev, nullable) [batch+1] receives the row offsets of each sequence.
 * host_upper_bound_rows (host, nullable) receives a bound on the row count known from the schedule
 * without reading the device (exact except for Greedy, whose windows may clip or overlap, and for
 * shifted logits). `step` must be the context's next step, else DKV_E_BAD_STATE.
 * Calling it is optional: dkv_denoise_step does it when it has not been done for that step. */
int dkv_select_active(dkv_ctx *ctx, int32_t step, int32_t *active_idx, int32_t *active_off,
                      int32_t *host_upper_bound_rows);

/* One denoising step (Algorithm 1 plus the unmasking of Sec. 3.1): embed the active rows, per
 * layer project Q/K/V, rotate, overwrite the rows' K/V in the cache, attend over all positions,
 * output projection, feed-forward; then final norm, vocabulary logits, softmax confidence and
 * arg max (MASK excluded, lowest id on ties) for the candidate rows (active, masked, in the
 * current block), and commit k positions per sequence: the most confident (ties to the lower
 * position) or the next entries of `order`.
 * forced_pos / forced_tok (dev, nullable, [batch, k]): commit these instead (teacher forcing);
 * each forced position must be a candidate of the step. logits_out (dev, nullable) receives the
 * fp32 logits of the candidate rows, [n_candidates, vocab], candidates ordered like the rows.
 * `step` must be the context's next step; the counter advances by one. */
int dkv_denoise_step(dkv_ctx *ctx, int32_t step, const int32_t *forced_pos,
                     const int32_t *forced_tok, float *logits_out);

/* Make the next step recompute the given scope whatever the schedule says (the cache refresh of
 * Sec. 3.3 on demand; also the way to rebuild a cache from tokens and mask alone). */
int dkv_refresh(dkv_ctx *ctx, int32_t scope);

/* Debug reads; each synchronises the stream. Sizes are capacities of the (host) outputs.
 * dkv_read_rows: active set of the last selected step: positions and offsets [batch+1].
 * dkv_read_candidates: candidates of the last executed step: position, predicted token,
 *   confidence, and offsets [batch+1].
 * dkv_read_hidden: the residual stream of the last executed step, [rows, d_model] fp32, at a layer
 *   boundary: `layer` = l in [0, n_layers) is the input of block l (l = 0: the embedded rows), `layer` =
 *   n_layers the output of the last block (before the final norm). The input of block l together with
 *   the cache rows of layer l is everything one block of Algorithm 1 (lines 3-6) consumes, so a single
 *   layer can be checked on its own at any step. Only `layer` = n_layers is kept by default; the other
 *   boundaries are available when dkv_capture_hidden was active during the step, else
 *   DKV_E_BAD_STATE. */
int dkv_read_rows(dkv_ctx *ctx, int32_t *pos, int32_t *off, int32_t capacity, int32_t *n_rows);
int dkv_read_candidates(dkv_ctx *ctx, int32_t *pos, int32_t *tok, float *conf, int32_t *off,
                        int32_t capacity, int32_t *n_cand);
int dkv_read_hidden(dkv_ctx *ctx, int32_t layer, float *out, int32_t capacity_rows, int32_t *n_rows);

/* Debug: from the next step on, every denoising step also copies the residual stream at each layer
 * boundary into `buffer` (dev), laid out [n_layers + 1][batch * seq_len][d_model] fp32 (slot l = input
 * of block l, slot n_layers = output of the last block; only the step's rows of each slot are written).
 * `bytes` is the buffer's size: DKV_E_INVALID_ARG if smaller than that layout. buffer = NULL stops the
 * copies. The buffer is caller-owned and must stay valid while capturing. */
int dkv_capture_hidden(dkv_ctx *ctx, float *buffer, size_t bytes);

int dkv_destroy(dkv_ctx *ctx);

/* Per-kernel timing for roofline reports. Between dkv_profile_begin and dkv_profile_end every
 * launch of a projection or attention kernel made by dkv_denoise_step is bracketed by HIP events on
 * the context's stream. dkv_profile_end synchronises the stream and fills `out` (host, array of
 * DKV_PROF_KINDS entries) with, per kernel kind: number of launches, summed duration in
 * milliseconds, and summed algorithmic bytes and flops of those launches:
 *   projection  bytes = (M*K + N*K) * sizeof(element) + output bytes   flops = 2*M*N*K
 *               (output: 4*M*N; M*(N/2)*sizeof(element) for gate/up with the fused SwiGLU; 0 for the
 *               vocabulary projection, whose epilogue keeps the softmax statistics only)
 *   attention   bytes = (2*batch*n_kv_heads*seq_len + 2*rows*n_q_heads) * head_dim * sizeof(element)
 *               flops = 4*rows*n_q_heads*seq_len*head_dim
 * with M the schedule's row count of the step. Kinds: */
#define DKV_GEMM_DMA_32x128   0   /* projection kernels by workgroup tile (rows x columns) */
#define DKV_GEMM_DMA_64x128   1
#define DKV_GEMM_DMA_128x128  2
#define DKV_GEMM_DMA_128x256  3
#define DKV_GEMM_DMA_256x256  4
#define DKV_GEMM_DMA_128x96   5
#define DKV_GEMM_DMA_128x192  6
#define DKV_GEMM_DMA_256x192  7
#define DKV_GEMM_DMA_192x256  8
#define DKV_GEMM_REG_64x128   9   /* bf16 with K not a multiple of 64 */
#define DKV_GEMM_SIMT         10  /* fp32 mode / generic */
#define DKV_PROF_ATTN         11  /* attention (including the key-slice merge when it runs) */
#define DKV_PROF_STREAM       12  /* projection kernels without a number of their own: the 256-row tiles that the library
                                     plans by itself for 129 to 256 rows inside a step */
#define DKV_PROF_KINDS        13
typedef struct {
    int64_t launches;
    double ms, bytes, flops;
} dkv_prof_entry;
int dkv_profile_begin(dkv_ctx *ctx);
int dkv_profile_end(dkv_ctx *ctx, dkv_prof_entry *out);

/* Text of the last error raised on the calling thread ("" if none). Never NULL. */
const char *dkv_last_error(void);

/* The cache update and attention of one layer in isolation (Algorithm 1 lines 4-6 in a
 * position-indexed layout; Eq. 4): for every active row r of sequence b at position
 * p = active_idx[r], k_cache[b][:, p, :] = k_new[r], v_cache[b][:, p, :] = v_new[r]; then
 * out[r, h, :] = softmax(q[r, h] . K[b][h / group]^T / sqrt(head_dim)) V[b][h / group] over ALL
 * seq_len positions, no mask.
 * All (dev): k_cache, v_cache [batch][n_kv_heads][seq_len][head_dim]; q, out [rows][n_q_heads]
 * [head_dim]; k_new, v_new [rows][n_kv_heads][head_dim]; active_idx [rows] (positions, distinct
 * within a sequence); active_off [batch+1]. `rows` (host) = active_off[batch];
 * `max_rows_per_seq` (host) bounds the rows of any one sequence (pass `rows` if unknown). Elements
 * of `dtype`. workspace (dev) of dkv_attn_update_workspace_bytes(...) bytes for the same bound. */
size_t dkv_attn_update_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                       int32_t seq_len, int32_t head_dim, int32_t dtype,
                                       int32_t max_rows_per_seq);
int dkv_attn_update(void *k_cache, void *v_cache, const void *q, const void *k_new,
                    const void *v_new, const int32_t *active_idx, const int32_t *active_off,
                    void *out, int32_t rows, int32_t max_rows_per_seq, int32_t batch,
                    int32_t n_q_heads, int32_t n_kv_heads, int32_t seq_len, int32_t head_dim,
                    int32_t dtype, void *workspace, size_t workspace_bytes, void *stream);

/* dkv_attn_update for callers that cannot allocate device memory or pass a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc. Same arguments, same kernels and the same
 * result as dkv_attn_update, but the scratch of key-sliced attention (partial softmax records) is a
 * DKV_STATIC_SCRATCH_BYTES array inside the library's device image; the call allocates nothing. Shapes whose
 * scratch (dkv_attn_update_workspace_bytes) exceeds that size are run with key slices that fit (the same result up
 * to the order of its sums). Each GPU holds one such array for the life of the process and all calls on that GPU share it:
 * calls that overlap on one GPU (different streams or threads) race on it; calls on one stream are ordered.
 * Nothing in the array needs clearing between calls. The first call on a device looks the array up and must
 * not happen inside a graph capture. */
#define DKV_STATIC_SCRATCH_BYTES (4u << 20)
int dkv_attn_update_static(void *k_cache, void *v_cache, const void *q, const void *k_new,
                           const void *v_new, const int32_t *active_idx, const int32_t *active_off,
                           void *out, int32_t rows, int32_t max_rows_per_seq, int32_t batch,
                           int32_t n_q_heads, int32_t n_kv_heads, int32_t seq_len, int32_t head_dim,
                           int32_t dtype, void *stream);

/* The paper's own cache operator, concat_reorder (Appendix A; Algorithm 1 lines 4-5), on its compact
 * layout: per (sequence, kv head) the n_cached cached rows and the n_new freshly computed rows are
 * concatenated and row i of the result is row take[b][i] of that concatenation (the order that puts the next
 * step's cached positions first). Not on this library's path (the position-indexed cache never moves);
 * exported so that what the layout choice saves can be measured on the same shapes.
 * All (dev): k_cached, v_cached [batch][n_kv_heads][n_cached][head_dim]; k_new, v_new [batch][n_kv_heads]
 * [n_new][head_dim]; take [batch][n_cached + n_new], a permutation of 0 .. n_cached + n_new - 1 per
 * sequence (values are not checked); k_out, v_out [batch][n_kv_heads][n_cached + n_new][head_dim], must not
 * overlap the inputs. head_dim * element size must be a multiple of 16. */
int dkv_concat_reorder(const void *k_cached, const void *v_cached, const void *k_new, const void *v_new,
                       const int32_t *take, void *k_out, void *v_out, int32_t batch, int32_t n_kv_heads,
                       int32_t n_cached, int32_t n_new, int32_t head_dim, int32_t dtype, void *stream);

/* A K/V cache in pages, for sequences of different lengths that grow and leave: position p of sequence b lives in page
 * page_table[b][p / page_size] at slot p % page_size. An entry outside [0, n_pages) says that there is no page: rows are not
 * stored there, loads give zeros, attention leaves those positions out (a table can be wider than what is in use, and a
 * page can be given back before its sequence ends). Pages may be shared by sequences that only read them.
 *   k_pages, v_pages (dev) [n_pages][n_kv_heads][page_size][head_dim], elements of `dtype`, 16-byte aligned; DKV_E2M1: two to a byte
 *                    ([head_dim / 2]), the lower dim in the lower 4 bits: a sign bit and 0, 0.5, 1, 1.5, 2, 3, 4 or 6
 *   k_scale, v_scale (dev) [n_pages][n_kv_heads][page_size], DKV_E4M3 only: scale of a row as the biased exponent of a
 *                    power of two (E8M0): element = code * 2^(scale - 127), of 17 to 247, which are those that a store writes; what
 *                    is read from a row with another one is not defined. DKV_E2M1: [n_pages][n_kv_heads][page_size][head_dim / 32], one for
 *                    each 32 dims, of 17 to 253, or 255, which makes the 32 dims NaN
 *   page_table (dev) [batch][max_pages]
 *   seq_len (dev) [batch] positions of each sequence (attention only; taken as 0 below 0, as max_pages * page_size above)
 * page_size: a power of two, 16 to 65536; max_pages * page_size at most 2^30, n_pages * n_kv_heads * page_size at most 2^32, n_kv_heads * head_dim
 * below 2^31; head_dim 32, 64 or 128; dtype DKV_BF16, DKV_FP32, DKV_E4M3 or DKV_E2M1. Nothing in the structure is kept by a call; the structure itself is host memory. Table, lengths, positions
 * and row offsets are read on the device, so a captured call follows them. The current device is that of the cache and the stream. */
typedef struct {
    void *k_pages, *v_pages;
    uint8_t *k_scale, *v_scale;
    const int32_t *page_table, *seq_len;
    int32_t batch, n_pages, max_pages, page_size, n_kv_heads, head_dim, dtype;
} dkv_paged_cache;

/* Write rows into the cache: row r of sequence b, i.e. row_off[b] <= r < row_off[b + 1], goes to position positions[r] of that
 * sequence. Rows whose position is negative, beyond the table or on no page are not stored, nor are rows from
 * min(rows, row_off[batch]) on. Positions are distinct within a sequence, and no page that two sequences share is written.
 *   k_new, v_new (dev) [rows] rows of [n_kv_heads][head_dim], `row_stride` elements apart (at least n_kv_heads * head_dim),
 *                elements of `dtype` (DKV_BF16 or DKV_FP32)
 *   positions (dev) [rows]; row_off (dev) [batch + 1] ascending from 0, or null for one row per sequence (rows == batch)
 * DKV_BF16 and DKV_FP32 caches hold the nearest value of their type. A DKV_E4M3 cache holds x * 2^-e rounded to the nearest e4m3
 * value, ties to even, with the smallest e >= -110 that brings the largest finite magnitude of the row to at most 448: an
 * error of at most 2^-4 of the element or 2^(e - 10), whichever is larger. Infinities and NaN become NaN, and count for nothing in e. (e is at
 * most 120, and then magnitudes end at 240 * 2^120, so that no finite element is read back as infinity.)
 * A DKV_E2M1 cache holds x * 2^-e rounded to the nearest of its values, ties to the even code, with the smallest e >= -110 that brings the largest
 * magnitude of the 32 dims to at most 6: an error of at most 2^-2 of the element or 2^(e - 2), whichever is larger. Where one of them is an infinity
 * or a NaN all 32 become NaN. (e is at most 126, and then magnitudes end at 3 * 2^126.)
 * What that costs attention: on normally distributed rows its result is off by 0.17 (relative, all elements together) of that over the rows before they were
 * stored, 0.3 where queries are three times as large and few keys count; DKV_E4M3 0.04 and 0.07, DKV_BF16 0.0025 and 0.0045. */
int dkv_paged_store(const dkv_paged_cache *cache, const void *k_new, const void *v_new, int64_t row_stride,
                    const int32_t *positions, const int32_t *row_off, int32_t rows, int32_t dtype, void *stream);

/* The inverse: k_out[r], v_out[r] (dev, [rows][n_kv_heads][head_dim] of `dtype`, DKV_BF16 or DKV_FP32) = the rows at positions[r],
 * zeros where the position is outside the table or on no page. Rows from min(rows, row_off[batch]) on are left as they
 * are. Exact, but for a DKV_FP32 cache read as DKV_BF16 (nearest value). */
int dkv_paged_load(const dkv_paged_cache *cache, void *k_out, void *v_out, const int32_t *positions,
                   const int32_t *row_off, int32_t rows, int32_t dtype, void *stream);

/* Attention of new rows over the cache (Eq. 4 with lengths of their own): for row r of sequence b and query head h
 *   out[r][h] = softmax(q[r][h] . K[b][h / group]^T / sqrt(head_dim)) V[b][h / group]
 * over the positions below seq_len[b] that lie on a page, no further mask. Where the sum of the exponentials is zero (no such position,
 * or all scores -infinity) the result is zero. What lies behind a sequence's end or on pages that the table does not name is
 * never used, whatever it holds.
 *   q (dev) [rows] rows of [n_q_heads][head_dim], `q_stride` elements apart (at least n_q_heads * head_dim); out (dev)
 *     [rows][n_q_heads][head_dim]; elements of `dtype`
 *   row_off as above; max_rows_per_seq (host) bounds the rows of any one sequence (rows of a sequence beyond it are left out); rows is at most
 *     batch * max_rows_per_seq, a larger one is refused
 *   workspace (dev), 16-byte aligned, of dkv_paged_attn_workspace_bytes for the same cache and heads and at least as many rows and as large a
 *     bound; calls that may overlap need one each
 * out overlaps none of the inputs. Results are finite where the sum of the magnitudes of V over a sequence's keys is below 2^128 (DKV_E4M3 and
 * DKV_E2M1: 2^120; the sums are divided last).
 * Rows from min(rows, row_off[batch]) on are left as they are. Kernels and slices are planned from the table's width, as if all of it were in
 * use: a call whose table is much wider than its lengths may take longer than with a narrow one, with the same results but for the order of sums.
 * dtype DKV_BF16 reads DKV_BF16, DKV_E4M3 and DKV_E2M1 caches (products of bf16 operands, probabilities among them, sums in fp32; e4m3 and e2m1
 * elements with their scales are exact in bf16); DKV_FP32 reads DKV_FP32, DKV_E4M3 and DKV_E2M1 caches, in fp32 throughout. */
size_t dkv_paged_attn_workspace_bytes(const dkv_paged_cache *cache, int32_t n_q_heads, int32_t rows, int32_t max_rows_per_seq,
                                      int32_t dtype);
int dkv_paged_attn(const dkv_paged_cache *cache, const void *q, int64_t q_stride, const int32_t *row_off, void *out,
                   int32_t rows, int32_t max_rows_per_seq, int32_t n_q_heads, int32_t dtype, void *workspace,
                   size_t workspace_bytes, void *stream);

/* Page tables that follow the lengths of their sequences. One set of tables serves the caches of all layers.
 *   page_table (dev) [batch][max_pages], seq_len (dev) [batch]: as in dkv_paged_cache
 *   free_pages (dev) [n_pages]: a ring of the numbers of the free pages; free_at (dev) [2]: the place of the first of them, and how many
 *                    there are. A cache without sequences has free_pages = 0 .. n_pages - 1, free_at = {0, n_pages} and seq_len = 0.
 * page_size, max_pages as in dkv_paged_cache; at most 2^30 pages, 2^20 sequences, and fewer than 2^31 entries of a table. Nothing is kept by a call. */
typedef struct {
    int32_t *page_table, *seq_len, *free_pages, *free_at;
    int32_t batch, n_pages, max_pages, page_size;
} dkv_paged_tables;

/* Give the sequences new lengths (dev) [batch]; a length below zero or beyond the table leaves its sequence as it is.
 * A sequence that gets longer takes pages for the positions behind its last page from the front of the ring, the first sequence first. They are those that were free
 * before the call: what it gives back can be taken by the next one. From the first sequence on for which they do not last, or the rows below do not, no sequence
 * gets longer; seq_len (and row_off) say which have.
 * A sequence that gets shorter gives the pages behind its new length back, to the end of the ring in the order of sequences and positions;
 * their entries become -1. (Entries that name no page are passed over. No two sequences may share what one of them gives back.)
 * Where row_off is not null the new positions are listed, as dkv_paged_store, dkv_rope and dkv_paged_attn take them:
 *   row_off (dev) [batch + 1]; positions (dev, nullable) [rows]; slots (dev, nullable) [rows]: page * page_size + slot of the position, -1 where
 *   the table names no page (a page given back before is not replaced while its sequence goes on)
 * Entries of positions and slots from row_off[batch] on are left as they are. rows is at most 2^30.
 * workspace (dev), 16-byte aligned, of dkv_paged_resize_workspace_bytes(batch) bytes; calls that may overlap need one each. Results do not depend
 * on timing. Tables, lengths and ring are read and changed on the device, so a captured call follows them. */
size_t dkv_paged_resize_workspace_bytes(int32_t batch);
int dkv_paged_resize(const dkv_paged_tables *tables, const int32_t *lengths, int32_t *row_off, int32_t *positions, int64_t *slots,
                     int32_t rows, void *workspace, size_t workspace_bytes, void *stream);

/* Rotary positions: each pair (a, b) of the first rot_dim dims of a head becomes scale * (a cos t - b sin t, b cos t + a sin t), t = position * freq[i],
 * pair i being the dims i and i + rot_dim / 2, or where `interleaved` 2 i and 2 i + 1. head_dim 32, 64 or 128; rot_dim even, 2 to head_dim; freq in
 * radians, rot_dim / 2 of them. Host memory, which dkv_rope_init fills and a caller may fill otherwise. */
typedef struct {
    int32_t head_dim, rot_dim, interleaved;
    float scale;
    double freq[64];
} dkv_rope_desc;

/* freq[i] = f = theta^(-2 i / rot_dim) and scale = 1, or, for longer contexts than a model was trained on:
 *   DKV_ROPE_LINEAR  f / factor
 *   DKV_ROPE_BASE    f of a larger base, theta * factor^(rot_dim / (rot_dim - 2)): the last pair is stretched by `factor`, the first not
 *   DKV_ROPE_PARTS   f * y + f / factor * (1 - y) with y = (original f / 2 pi - slow) / (fast - slow) within [0, 1]: pairs that turn at least
 *                    `fast` times over `original` positions stay, those that turn at most `slow` times are stretched; scale = 0.1 ln(factor) + 1.
 *                    y is linear in the number of turns; a model that was trained with one that is linear in the pair's index i has to set freq
 * original, slow and fast are read for DKV_ROPE_PARTS only (usual: slow 1, fast 32), factor not for DKV_ROPE_NONE. */
#define DKV_ROPE_NONE   0
#define DKV_ROPE_LINEAR 1
#define DKV_ROPE_BASE   2
#define DKV_ROPE_PARTS  3
int dkv_rope_init(dkv_rope_desc *rope, int32_t head_dim, int32_t rot_dim, int32_t interleaved, double theta, int32_t scaling,
                  double factor, double original, double slow, double fast);

/* Rotate the rows of q and k by their positions:
 *   q, k (dev) [rows] rows of [n_q_heads][head_dim] and [n_k_heads][head_dim], `q_stride` and `k_stride` elements apart (at least a row);
 *     q_out, k_out the same with strides of their own: the inputs themselves (then with their stride), or memory that overlaps neither input.
 *     n_q_heads or n_k_heads may be 0. Dims from rot_dim on are copied. Elements of `dtype` (DKV_BF16 or DKV_FP32), rounded once.
 *   positions (dev) [rows]; row_off (dev, nullable) [batch + 1]: rows from row_off[batch] on are left as they are
 * `inverse`: t = -position * freq[i], with the same scale: the gradient of q and k from that of q_out and k_out.
 * Angles are formed in 64 bits, so that far positions lose nothing. */
int dkv_rope(const dkv_rope_desc *rope, const void *q, int64_t q_stride, void *q_out, int64_t q_out_stride, int32_t n_q_heads,
             const void *k, int64_t k_stride, void *k_out, int64_t k_out_stride, int32_t n_k_heads, const int32_t *positions,
             const int32_t *row_off, int32_t batch, int32_t rows, int32_t dtype, int32_t inverse, void *stream);

/* y[M, N] (fp32, dev) = x[M, K] * w[N, K]^T with x, w of `dtype` (dev): the projection kernel of
 * the path on its own, for parity tests and roofline measurements. workspace as returned by
 * dkv_gemm_workspace_bytes. */
size_t dkv_gemm_workspace_bytes(int32_t m, int32_t n, int32_t k, int32_t dtype);
int dkv_gemm(const void *x, const void *w, float *y, int32_t m, int32_t n, int32_t k,
             int32_t dtype, void *workspace, size_t workspace_bytes, void *stream);
/* The same with the kernel (DKV_GEMM_*), the number of K slices and the launch options chosen by the
 * caller instead of the library's heuristic, so every kernel can be checked on every shape. workspace
 * must hold split_k * m * n floats when split_k > 1. `options` is a sum of DKV_GEMM_OPT_* (ignored by
 * the kernels that have no such option, and dropped when the grid does not fit them).
 * DKV_E_UNSUPPORTED if the kernel does not take the shape, DKV_E_INVALID_ARG for unknown option bits. */
#define DKV_GEMM_OPT_STAGGER    1   /* every workgroup starts its K loop at a different K tile */
#define DKV_GEMM_OPT_XCD_GROUP  2   /* workgroups that share an XCD's L2 take neighbouring tiles */
#define DKV_GEMM_OPT_STREAM_W   8   /* weights fetched with the non-temporal hint (dropped with more than one row of tiles;
                                       the 192x256, 256x192 and 256x256 tiles have no such loads) */
#define DKV_GEMM_OPT_SWIGLU     4   /* fused SwiGLU epilogue: w rows are gate_0, up_0, gate_1, up_1, ...; y is then
                                       a `dtype` (bf16) array [M, N/2] with y[m][j] = silu(x w_{2j}) * (x w_{2j+1});
                                       tile kernels with split_k == 1 only, else DKV_E_UNSUPPORTED */
int dkv_gemm_with(const void *x, const void *w, void *y, int32_t m, int32_t n, int32_t k,
                  int32_t dtype, int32_t kind, int32_t split_k, int32_t options, void *workspace,
                  size_t workspace_bytes, void *stream);

/* Yardsticks for roofline reports, not part of the path: what the chip sustains for a plain copy (the kernel
 * HBM byte counters are calibrated with), a streaming read, and a register-only dense bf16 MFMA loop. All
 * (dev) buffers; `bytes` a multiple of 16; sink: at least 2 MiB, never written in practice. dkv_peak_mfma stores
 * the flops of its launch in *flops (host). The caller times the launches on `stream`. */
int dkv_peak_copy(const void *src, void *dst, size_t bytes, void *stream);
int dkv_peak_read(const void *src, void *sink, size_t bytes, void *stream);
int dkv_peak_mfma(void *sink, int32_t iters, double *flops, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DKV_H */
