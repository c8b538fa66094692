/*
 * knnssd.h - C ABI of the MI355X-native KNN-SSD decode path.
 *
 * KNN-SSD (paper Sec. 4): a decoder-only LLM M with L = 2*n_blocks skippable
 * sublayers (attention and MLP counted separately, Sec. 3.1) drafts tokens with
 * a subset of its own sublayers, M(z), and verifies them with the full model in
 * one forward pass (Sec. 4.2). Which skip set z is used is decided per sample
 * by a nearest-neighbour search of the prompt's last hidden vector among stored
 * anchor vectors (Sec. 4.2, Eq. 4-6). Decoding is greedy, so the emitted tokens
 * are exactly the full model's own greedy continuation (Sec. 3.1).
 *
 * Conventions
 *   - "dev" pointers are device (HBM) addresses, "host" pointers host addresses.
 *   - The caller owns every device buffer (weights, KV cache, workspace, anchor
 *     table) and the HIP stream; the library allocates no device memory. All
 *     buffers must stay valid until knnssd_destroy.
 *   - Every matrix is given row-major [out_features][in_features]; weight_dtype says
 *     whether matrices hold fp32 or bf16 values. RMSNorm gains are always fp32. For the
 *     tuned bf16 kernels the caller repacks each matrix once into stream order
 *     (knnssd_pack_matrix) and sets cfg.weights_packed.
 *   - Skip mask layout: mask[2*b] = 1 skips the attention sublayer of block b,
 *     mask[2*b+1] = 1 skips its MLP sublayer (z_i = 1 means "skip", Sec. 3.1).
 *   - Activations, residual stream, RoPE, softmax and all accumulators are fp32;
 *     keys/values are rounded to kv_dtype (nearest-even) when they are cached.
 *   - Every call returns KNNSSD_OK (0) or a negative error code. Arguments are
 *     validated before anything is launched. Calls are synchronous with respect
 *     to their host outputs (the stream is drained before scalars are returned).
 *     A context is not thread-safe.
 */
#ifndef KNNSSD_H
#define KNNSSD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KNNSSD_OK 0
#define KNNSSD_EINVAL (-1)      /* null pointer or malformed argument                     */
#define KNNSSD_ESHAPE (-2)      /* shape not supported by the kernels                     */
#define KNNSSD_ERANGE (-3)      /* position / length / token id outside the valid range   */
#define KNNSSD_EDEGENERATE (-4) /* zero-norm or non-finite query / anchor (cosine undefined) */
#define KNNSSD_ESTATE (-5)      /* call made in the wrong order                           */
#define KNNSSD_EHIP (-6)        /* a HIP runtime call failed                              */

#define KNNSSD_FP32 0
#define KNNSSD_BF16 1

#define KNNSSD_PREFILL_AUTO 0
#define KNNSSD_PREFILL_CHUNKED 1
#define KNNSSD_ATTN_MFMA 0
#define KNNSSD_ATTN_VALU 1
#define KNNSSD_MERGE_FUSED 0
#define KNNSSD_MERGE_SEPARATE 1

#define KNNSSD_MAX_ROWS 16  /* rows one verification pass can carry: max_draft + 1 <= 16 */

typedef struct knnssd_model_cfg {
    int32_t n_blocks, d_model, n_heads, n_kv_heads, head_dim, d_ffn, vocab;
    int32_t max_seq;      /* KV-cache capacity in positions                          */
    int32_t max_anchors;  /* largest anchor table knnssd_set_anchors will be given   */
    float rope_base;      /* RoPE: rotate-half pairs (i, i+head_dim/2), angle pos*base^(-2i/head_dim) */
    float rms_eps;
    int32_t weight_dtype; /* KNNSSD_FP32 | KNNSSD_BF16 */
    int32_t kv_dtype;     /* KNNSSD_FP32 | KNNSSD_BF16 */
    int32_t weights_packed; /* 1: wqkv/wo/wgu/wdown/lm_head are in stream order (knnssd_pack_matrix) and the
                               tuned bf16 kernels run; 0: row-major, generic kernels. embed is always row-major. */
    int32_t prefill_mode;   /* KNNSSD_PREFILL_AUTO: prompts go through the many-row prefill kernels where the shape
                               fits them; KNNSSD_PREFILL_CHUNKED: through 16-row passes of the verification kernels.
                               Row-major weights: AUTO takes a prompt's rows side by side where that is faster, with the
                               bits of 16-row passes, if the workspace has room for them (knnssd_workspace_bytes of that cfg). */
    int32_t verify_attn;    /* which split-KV attention kernel verification passes (and the draft steps of
                               grouped-query models, and of any model once the context brings more (kv head,
                               256-position chunk) items than 512) use: KNNSSD_ATTN_MFMA (matrix cores, the default) or
                               KNNSSD_ATTN_VALU (vector ALUs). One kernel per context, never chosen per pass, so a
                               row's result does not depend on how many rows share its pass. Only read with
                               weights_packed = 1. Results stay within the stated tolerances either way. */
    int32_t attn_merge;     /* where the chunks of the split-KV attention are merged: KNNSSD_MERGE_FUSED (the default:
                               inside the attention launch, by the workgroup that finishes a group's last chunk, while
                               a kv head has at most four (row, head) pairs and the context at most 2048 positions
                               (6144 on the matrix-core kernel); in a launch of its own beyond) or
                               KNNSSD_MERGE_SEPARATE (always in a launch of its own). Same arithmetic, same bits.
                               Only read with weights_packed = 1. */
} knnssd_model_cfg;

/* Device pointers to the model. The four per-block members are HOST arrays of
 * n_blocks DEVICE pointers (the arrays are copied by knnssd_create).
 *   wqkv[b]  : [(n_heads + 2*n_kv_heads)*head_dim][d_model]  rows: all q heads, then k heads, then v heads
 *   wo[b]    : [d_model][n_heads*head_dim]
 *   wgu[b]   : [2*d_ffn][d_model]                            rows: gate rows, then up rows
 *   wdown[b] : [d_model][d_ffn]                                                            */
typedef struct knnssd_weights {
    const void *embed;          /* [vocab][d_model] */
    const void *lm_head;        /* [vocab][d_model] */
    const float *final_norm;    /* [d_model] */
    const float *const *attn_norm;
    const void *const *wqkv;
    const void *const *wo;
    const float *const *mlp_norm;
    const void *const *wgu;
    const void *const *wdown;
} knnssd_weights;

typedef struct knnssd_gen_cfg {
    int32_t max_new;       /* tokens to emit after the prompt (the prefill's own token included) */
    int32_t max_draft;     /* K: draft tokens per round, 0 = plain autoregressive decoding, <= 15 */
    float conf_threshold;  /* > 0: stop drafting after the first draft whose top-1 probability is
                              below it (that token is still verified); <= 0 disables the rule    */
    int32_t keep_mask;     /* 1: do not route this sample, draft with the mask already installed (the
                              fixed-configuration Self-SD baseline of Sec. 5.1 on a task stream); 0: route */
} knnssd_gen_cfg;

/* Counters of one knnssd_generate call. Mean generated length M = (emitted-1)/rounds and
 * acceptance rate alpha = accepted/drafted are the paper's App. C.2 metrics. Times are GPU
 * time from HIP events on the context's stream; ns_draft, ns_verify: from the device's clock, a round's
 * draft steps from the end of the round before, its verification from there on (the two are the whole decode). */
typedef struct knnssd_stats {
    int64_t rounds, drafted, accepted, emitted;
    int64_t ns_prefill, ns_knn, ns_draft, ns_verify, ns_total;
    int64_t draft_passes, verify_passes;
} knnssd_stats;

typedef struct knnssd_ctx knnssd_ctx;

/* Stream order. The tuned kernels read each weight matrix once per pass, front to back, in the
 * order their wavefronts consume it; knnssd_pack_matrix rewrites a row-major bf16 matrix into
 * that order (same size, out of place, one kernel on hip_stream; src and dst are device
 * pointers, 16-byte aligned, and must not overlap). knnssd_pack_supported says whether a shape
 * can use it (bf16 weights and cache, d_model, d_ffn and n_heads*head_dim multiples of 32). */
#define KNNSSD_W_QKV 0      /* [(n_heads+2*n_kv_heads)*head_dim][d_model] */
#define KNNSSD_W_O 1        /* [d_model][n_heads*head_dim]                */
#define KNNSSD_W_GATE_UP 2  /* [2*d_ffn][d_model]                         */
#define KNNSSD_W_DOWN 3     /* [d_model][d_ffn]                           */
#define KNNSSD_W_LM_HEAD 4  /* [vocab][d_model]                           */
int32_t knnssd_pack_supported(const knnssd_model_cfg *cfg);
int32_t knnssd_pack_matrix(const knnssd_model_cfg *cfg, int32_t which, const void *src_dev, void *dst_dev,
                           void *hip_stream);

/* Bytes of device workspace / KV cache a context of this shape needs (0 if cfg is invalid). */
size_t knnssd_workspace_bytes(const knnssd_model_cfg *cfg);
size_t knnssd_kvcache_bytes(const knnssd_model_cfg *cfg);

/* Create a context over caller-owned device memory. kv_dev and ws_dev must be 256-byte
 * aligned; kv_bytes and ws_bytes are the sizes of the two buffers, and the call fails with
 * KNNSSD_EINVAL when either is smaller than the size queries above say for THIS cfg (the queries
 * depend on every field, weights_packed included). With KNNSSD_PREFILL_AUTO a workspace that lacks only the room
 * that makes prompts faster is accepted and prompts go without it: row-major weights take 16-row passes
 * (the size that KNNSSD_PREFILL_CHUNKED asks for is enough), stream-order ones the plain tiles of the prefill
 * kernels (at some sizes a third less than the query says). hip_stream is a hipStream_t (NULL = the null
 * stream). Launches a few set-up kernels (RoPE table, the workgroups' shares of each matrix) on the stream.
 * The library reads no environment variable: every switch is a cfg field. */
int32_t knnssd_create(const knnssd_model_cfg *cfg, const knnssd_weights *w, void *kv_dev, size_t kv_bytes,
                      void *ws_dev, size_t ws_bytes, void *hip_stream, knnssd_ctx **out);
int32_t knnssd_destroy(knnssd_ctx *ctx);

/* Anchor table for the KNN routing step (Sec. 4.1: anchors a_ij with their domain label i and
 * one stored skip set z*_i per domain). anchors_dev: [n_anchors][dim] in anchor_dtype (KNNSSD_FP32, or
 * KNNSSD_BF16: half the bytes to scan; the values the caller stored ARE the anchors, products and sums stay
 * fp32), 16-byte aligned, dim must equal d_model; labels_dev: int32 [n_anchors] in [0, n_domains); masks_host:
 * uint8 [n_domains][mask_len], copied; mask_len must be 2*n_blocks (KNNSSD_ESHAPE otherwise: the table is read
 * with that row length). n_anchors <= cfg.max_anchors. */
int32_t knnssd_set_anchors(knnssd_ctx *ctx, const void *anchors_dev, int32_t anchor_dtype, const int32_t *labels_dev,
                           int32_t n_anchors, int32_t dim, const uint8_t *masks_host, int32_t n_domains,
                           int32_t mask_len);

/* Prefill (Sec. 4.2: the routing query is the prompt's last hidden vector): the full model over
 * n prompt tokens at positions 0..n-1. Resets the KV cache length to n. Outputs: the first
 * generated token (host) and, if last_hidden_dev is not NULL, the final-RMSNorm hidden state of
 * the last prompt token (fp32 [d_model], device) - the vector the KNN step is queried with. How the sums over a row
 * are grouped follows n (the kernels are chosen by it), so the same first tokens in a longer prompt give the same
 * hidden states and cache entries to fp32 rounding, not bit for bit; the same call gives the same bits. */
int32_t knnssd_prefill(knnssd_ctx *ctx, const int32_t *tokens_host, int32_t n, float *last_hidden_dev,
                       int32_t *first_token_out);

/* Eq. 4-6: cosine-similarity arg-max of query_dev (fp32 [d_model], device) over all anchors
 * (lowest index wins a tie), domain = that anchor's label, and the domain's stored skip set
 * becomes the context's draft mask. Host outputs may be NULL. mask_out: 2*n_blocks bytes. */
int32_t knnssd_select_skipset(knnssd_ctx *ctx, const float *query_dev, int32_t *anchor_idx_out,
                              int32_t *domain_out, uint8_t *mask_out);

/* Install a draft mask directly (2*n_blocks bytes on the host; NULL = skip nothing). */
int32_t knnssd_set_skipset(knnssd_ctx *ctx, const uint8_t *mask_host);

/* K nearest anchors (cosine similarity: Eq. 4 generalised from the arg-max to the K best, lowest index first among
 * equal scores) of each of n_queries query vectors against the installed anchor table, and the majority domain
 * among the K (a tie between domains goes to the tied domain whose best anchor ranks first; K = 1 is Eq. 4-5).
 * Batched: up to 4 queries share one pass over the table. queries_dev: fp32 [n_queries][d_model], 16-byte aligned
 * (device). anchor_idx_out: int32 [n_queries][k] (host). cosine_out: fp32 [n_queries][k] (host, may be NULL).
 * domain_out: int32 [n_queries] (host). 1 <= k <= 16 and k <= number of anchors. Installs no mask.
 * KNNSSD_EDEGENERATE for a zero-norm or non-finite query or anchor, KNNSSD_ESTATE without an anchor table,
 * KNNSSD_ERANGE for k or n_queries out of range or a table of more than 2^24 anchors. */
#define KNNSSD_KNN_KMAX 16
int32_t knnssd_knn_topk(knnssd_ctx *ctx, const float *queries_dev, int32_t n_queries, int32_t k,
                        int32_t *anchor_idx_out, float *cosine_out, int32_t *domain_out);

/* The routing step for callers that cannot allocate device memory or hand over a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc. Same scan and arg-max kernels as
 * knnssd_select_skipset, no context: the per-anchor scores (the kernels' scratch buffer) live in a device array
 * inside the library (KNNSSD_ROUTE_MAX_ANCHORS floats = 256 KB on every GPU the library runs on, held until the
 * process ends); the call allocates and frees nothing and never waits for the GPU. Everything is enqueued on
 * hip_stream (a hipStream_t of the CURRENT device); result_dev (device, int32[4]) receives, in stream order:
 * [0] the arg-max anchor n* (lowest index on ties), [1] its label, [2] 1 if a zero-norm or non-finite query or
 * anchor was met (then [0] = [1] = -1), [3] the bits of the fp32 score (v . a) / |a|. query_dev: fp32 [dim];
 * anchors_dev: fp32 [n_anchors][dim]; labels_dev: int32 [n_anchors]; all device pointers, query and anchors 16-byte
 * aligned; dim a multiple of 4. KNNSSD_ERANGE when n_anchors is not in [1, KNNSSD_ROUTE_MAX_ANCHORS], KNNSSD_ESHAPE
 * for a bad dim, KNNSSD_EINVAL for null or misaligned pointers; nothing is enqueued on an error. All calls on one
 * GPU share that GPU's array: calls whose kernels may overlap on one GPU (different streams, no ordering between
 * them) race on it. */
#define KNNSSD_ROUTE_MAX_ANCHORS 65536
int32_t knnssd_route_static(const float *query_dev, const float *anchors_dev, const int32_t *labels_dev,
                            int32_t n_anchors, int32_t dim, void *hip_stream, int32_t *result_dev);

/* Anchor index n* and domain (Eq. 4-5) of the most recent routing on this context, whether it was made by
 * knnssd_select_skipset or inside knnssd_generate; both are -1 before the first routing. Either output
 * pointer may be NULL. Host-only, no device work. */
int32_t knnssd_last_selection(const knnssd_ctx *ctx, int32_t *anchor_idx_out, int32_t *domain_out);

/* One draft step (Eq. 7): token_in at position pos through M(z) with the installed mask; only
 * retained attention sublayers read and write the KV cache. Returns the arg-max token (lowest
 * index on ties) and its softmax probability at temperature 1. pos must be < max_seq and at most one past the
 * last position written so far (the prefill's and the accepted rows', plus the draft steps made since the last
 * verification): KNNSSD_ERANGE otherwise, since attention would read entries nobody wrote. */
int32_t knnssd_draft_step(knnssd_ctx *ctx, int32_t token_in, int32_t pos, int32_t *token_out,
                          float *top1_prob_out);

/* Verification (Sec. 4.2): the full model over n rows tokens_host = [x_last, d_1..d_k]
 * (n = k+1 <= KNNSSD_MAX_ROWS) at positions start_pos..start_pos+k in ONE pass; every block
 * overwrites its KV entries at those positions; row i attends to positions 0..start_pos+i.
 * Greedy acceptance: *n_accepted_out = j, the number of leading drafts equal to the model's own
 * token; *next_token_out = the model's token after the accepted prefix; *new_cache_len_out =
 * start_pos + j + 1 (cache entries beyond it are dead: rollback is this counter). start_pos must not exceed the
 * current cache length (KNNSSD_ERANGE): draft steps fill only the retained blocks' entries, so the full model
 * can only continue from positions that a prefill or a verification wrote. */
int32_t knnssd_verify(knnssd_ctx *ctx, const int32_t *tokens_host, int32_t n, int32_t start_pos,
                      int32_t *n_accepted_out, int32_t *next_token_out, int32_t *new_cache_len_out);

/* The whole per-sample path: prefill, KNN routing (query_dev, or the prompt's own last hidden
 * vector when query_dev is NULL; skipped when no anchor table is set or max_draft = 0, in which
 * case the installed mask is used), then draft/verify rounds until max_new tokens are out.
 * out_tokens_host must hold max_new entries; *n_out receives the count. n_prompt + max_new +
 * max_draft must not exceed max_seq. stats may be NULL. */
int32_t knnssd_generate(knnssd_ctx *ctx, const int32_t *prompt_host, int32_t n_prompt,
                        const float *query_dev, const knnssd_gen_cfg *gen, int32_t *out_tokens_host,
                        int32_t *n_out, knnssd_stats *stats);

/* Measurement aid: enqueues ONLY the launches of the weight-streaming kernel of one draft step
 * (kind 0, n = 1, the installed mask: gemv_kernel) or of one verification pass (kind 1,
 * n <= KNNSSD_MAX_ROWS rows: gemm_mfma_kernel), back to back on the context's stream between two
 * HIP events. Outputs: the number of launches, the GPU time between the events (ns, in both
 * gemm_ns and pass_ns) and the weight bytes the launches streamed, so bytes / time is the
 * kernel's achieved bandwidth and time / launches its average duration. The pass's other
 * kernels are skipped, so its numerical outputs are meaningless and the cache entries at
 * start_pos.. are overwritten: prefill again before decoding. KNNSSD_ESHAPE if the shape runs on
 * the generic kernels. */
int32_t knnssd_profile_pass(knnssd_ctx *ctx, int32_t kind, const int32_t *tokens_host, int32_t n, int32_t start_pos,
                            int64_t *n_launches, int64_t *gemm_ns, int64_t *gemm_bytes, int64_t *pass_ns);

/* How the passes of small any-shape models (matrices of at most 8 MB a block and in the head) are put on the stream:
 * KNNSSD_PASS_AUTO (the default) chooses between one launch for the whole pass and a launch per step, KNNSSD_PASS_LAUNCHES
 * takes the latter always, KNNSSD_PASS_ONE the former wherever the pass fits it. Other models always run as a launch per step.
 * The workgroups of a one-launch pass wait for each other for a bounded time; if that runs out (they are not on the GPU
 * together) the last one runs the pass by itself, and KNNSSD_PASS_AUTO goes back to launches for a while. Test aid: workgroup quit_workgroup (KNNSSD_QUIT_ALL: every one,
 * KNNSSD_QUIT_ALONE: also the one that runs the pass by itself, which makes the call fail with KNNSSD_EHIP; -1: none) gives up
 * at its first wait from block quit_block on (n_blocks: the LM head's). */
#define KNNSSD_PASS_AUTO 0
#define KNNSSD_PASS_LAUNCHES 1
#define KNNSSD_PASS_ONE 2
#define KNNSSD_QUIT_ALL 64
#define KNNSSD_QUIT_ALONE 65
int32_t knnssd_set_pass_mode(knnssd_ctx *ctx, int32_t mode, int32_t quit_workgroup, int32_t quit_block);

/* One-launch passes of this context so far, and those of them that were broken up. */
int32_t knnssd_pass_counts(knnssd_ctx *ctx, int64_t *one_launch_out, int64_t *broken_up_out);

/* Parity/debug: fp32 logits of row `row` of the most recent pass (draft: row 0). */
int32_t knnssd_get_logits(knnssd_ctx *ctx, int32_t row, float *logits_host);

/* Parity/debug: cached key and value (as fp32) of one block at one position,
 * each [n_kv_heads*head_dim] on the host. */
int32_t knnssd_read_kv(knnssd_ctx *ctx, int32_t block, int32_t pos, float *k_host, float *v_host);

/* One transition of the task stream of Sec. 4.2, Eq. 8 (host only, no device work): the next sample stays in domain
 * `current` unless u_switch < mix_ratio; on a switch it lands on one of the other n_domains - 1 domains, taken in
 * increasing order, chosen by u_pick. u_switch and u_pick are uniform draws on [0, 1) the caller supplies (the library
 * draws no random numbers). Returns the next domain, or KNNSSD_EINVAL / KNNSSD_ERANGE (negative) for n_domains < 1, a
 * current domain outside [0, n_domains), a mix ratio outside [0, 1] or a draw outside [0, 1). */
int32_t knnssd_stream_next_domain(int32_t current, int32_t n_domains, double mix_ratio, double u_switch, double u_pick);

/* ---- Batches of requests over a paged cache --------------------------------------------------------------------
 * For callers that take several requests through a model at a time: their own program runs the matrix products, these
 * calls do what depends on which row belongs to which request. None of them needs a context, allocates memory or waits
 * for the GPU: everything is put on hip_stream (a stream of the CURRENT device) and may be captured into a HIP graph; the lengths
 * and tables are read on the device when the work runs, so that a replay follows what has been written there since. Arguments
 * are checked before anything is launched. What only the device knows is bounded there: a page id outside the cache, a
 * length beyond the table or a row beyond the batch gives wrong values in the rows concerned, never an access out of range.
 *
 * A batch is n_requests requests of which request r has cached[r] positions in the cache and added[r] new rows (tokens: a prompt, a
 * chunk of one, one token, or drafts to verify; 0 is allowed). The rows of all requests lie one behind the other:
 * request r's are row_start[r] .. row_start[r+1]-1, at positions cached[r], cached[r]+1, ... Rows behind the last
 * request's, if a buffer has any, are left as they were.
 *
 * One round of a batch: knnssd_page_plan (once), then for every block knnssd_paged_store and knnssd_paged_attention. Calls that
 * share tables, pages or a workspace have to be ordered (one stream, or events).                                       */
#define KNNSSD_MAX_REQUESTS 4096
#define KNNSSD_MAX_ROW_HEADS (1 << 25)      /* rows times query heads of an attention call; a quarter of it: requests times heads, rows of a store */

/* The keys and values of one block in pages. Position p of page g and kv head h begins at element
 * g*page_stride + h*head_stride + p*pos_stride of k_dev and of v_dev: [page][head][position][head_dim] and
 * [page][position][head][head_dim] are both such orders. Both bases and every stride times the element size are multiples of 16 bytes
 * (KNNSSD_EINVAL), strides are positive, pos_stride and head_stride at least head_dim. page_size is a power of two from 8 to 1024,
 * head_dim 64 or 128, n_pages * page_size at most 2^31 - 1, pos_stride at most 2^26 (KNNSSD_ESHAPE). */
typedef struct knnssd_pages {
    void *k_dev, *v_dev;
    int64_t page_stride, head_stride, pos_stride;       /* in elements */
    int32_t n_pages, page_size, n_kv_heads, head_dim, kv_dtype;
} knnssd_pages;

/* Which pages belong to whom, on the device. Request r holds the pages block_table[r][0 .. held[r]-1] for its positions
 * 0 .. held[r]*page_size-1; free_pages[0 .. *n_free-1] is a stack of the pages nobody holds (entries beyond are not looked at). A fresh
 * pool: held all 0, free_pages any permutation of the page ids, *n_free = n_pages. */
typedef struct knnssd_page_tables {
    int32_t *block_table_dev;   /* [n_requests][table_width] */
    int32_t *held_dev;          /* [n_requests] */
    int32_t *free_pages_dev;    /* [n_pages] */
    int32_t *n_free_dev;        /* [1] */
    int32_t n_requests, table_width, n_pages, page_size;
} knnssd_page_tables;

/* What the rows of one round are, on the device; all written by knnssd_page_plan. */
typedef struct knnssd_batch_rows {
    int32_t *row_start_dev;     /* [n_requests + 1] */
    int32_t *kv_len_dev;        /* [n_requests] cached + added */
    int32_t *slots_dev;         /* [max_rows] page * page_size + position in the page; -1 behind the last row */
    int32_t *positions_dev;     /* [max_rows] position in the request; -1 behind the last row */
    int32_t *result_dev;        /* [4] rows, pages taken minus pages given back, 0 or what was wrong (below), the longest kv_len */
    int32_t max_rows;
} knnssd_batch_rows;

/* Block tables and slots from the requests' lengths. Afterwards request r holds exactly ceil((cached[r] + added[r]) / page_size)
 * pages: those it no longer needs (rejected drafts, a finished request with cached = added = 0) go back to the stack and their
 * table entries become -1, then those it lacks are taken. The order is fixed: pages go back in descending order of request
 * and page and are taken in ascending order, so the same state and lengths give the same tables.
 * cached_dev or added_dev may be kv_len_dev itself (the lengths of the last round, all 0 after a round that could not be done).
 * result_dev[2] says in stream order whether it could be done: KNNSSD_PLAN_OK, or one of the following, the first that holds, and then tables and
 * stack are as they were, row_start and kv_len all 0, slots and positions all -1: the rest of the round does nothing.
 * KNNSSD_ERANGE for n_requests outside [1, KNNSSD_MAX_REQUESTS] or max_rows < 1, KNNSSD_ESHAPE for a page size or pool outside what knnssd_pages
 * allows or table_width < 1 or n_requests * table_width > 2^31 - 1. */
#define KNNSSD_PLAN_OK 0
#define KNNSSD_PLAN_MALFORMED 1     /* a negative length, or held / n_free outside what the tables can hold */
#define KNNSSD_PLAN_ROWS 2          /* more than max_rows rows */
#define KNNSSD_PLAN_WIDTH 3         /* a request needs more than table_width pages */
#define KNNSSD_PLAN_PAGES 4         /* the pool has too few pages */
int32_t knnssd_page_plan(const knnssd_page_tables *tables, const int32_t *cached_dev, const int32_t *added_dev,
                         const knnssd_batch_rows *rows, void *hip_stream);

/* Rotary embedding of a block's queries and keys, and its keys and values into the pages. qkv_dev: [n_rows] rows, qkv_stride elements
 * apart, of n_heads query heads, then the keys of the kv heads, then their values, head_dim values each (the rows of wqkv), in dtype. Pairs
 * (i, i + head_dim/2) are turned by position * rope_base^(-2i/head_dim): angles in 64 bits up to whole turns, the rest's sine and cosine and the products in fp32, one
 * rounding to what is stored. Rotated queries go to q_out_dev (NULL: nowhere), rotated keys also to k_out_dev (NULL: only into the pages),
 * both in dtype, rows q_out_stride / k_out_stride elements apart; either may lie over the same heads of qkv_dev. Keys and values go to
 * page slot / page_size, position slot % page_size, in the cache's type. A row whose slot is negative or outside the cache, or whose position is
 * negative, is skipped: nothing is written for it. No two rows may have the same slot. dtype KNNSSD_BF16 over an fp32 cache is refused
 * (KNNSSD_EINVAL). n_heads may be 0 (KNNSSD_ERANGE if negative, n_rows outside [1, KNNSSD_MAX_ROW_HEADS / 4], rope_base not positive and finite). Bases and strides as in knnssd_pages. */
int32_t knnssd_paged_store(const knnssd_pages *pages, const void *qkv_dev, int32_t dtype, int64_t qkv_stride, int32_t n_rows,
                           int32_t n_heads, const int32_t *slots_dev, const int32_t *positions_dev, float rope_base,
                           void *q_out_dev, int64_t q_out_stride, void *k_out_dev, int64_t k_out_stride, void *hip_stream);

/* Attention of the batch's new rows over the pages: row i of request r (n rows, length L = kv_len[r]) attends to positions
 * 0 .. L - n + i (none: its output is 0), with softmax(scale * q.k); query head h reads kv head h / (n_heads / n_kv_heads). q_dev, out_dev:
 * [n_rows] rows of n_heads * head_dim values in dtype, q_stride / out_stride elements apart; they must not overlap. dtype is
 * the cache's type, or KNNSSD_FP32 over a bf16 cache. Scores, softmax and sums are fp32; with dtype KNNSSD_BF16 the weights are rounded to
 * bf16 for the product with the values. Positions from kv_len on are not looked at; keys and values that a row does not see but a
 * later one of its request does have to be finite, and a row that sees an infinite value may have NaN where its output would be
 * infinite. Sums are of values times weights that may be more than 1: |value| times the positions of its request has to stay below
 * 2^96. block_table_dev: [n_requests][table_width]. most_rows: an upper bound of a request's rows if the caller has one, else 0; it only chooses the kernels. How the sums over a row are grouped follows the batch; the same call gives the
 * same bits. ws_dev: knnssd_paged_attention_bytes of the same pages, n_heads and dtype (0: not a supported shape), 256-byte aligned, of any
 * contents; nothing in it outlives a call.
 * KNNSSD_ESHAPE where n_heads is not a multiple of n_kv_heads, KNNSSD_ERANGE for n_requests outside [1, KNNSSD_MAX_REQUESTS], n_rows < 1,
 * n_rows * n_heads > KNNSSD_MAX_ROW_HEADS, n_requests * n_heads > KNNSSD_MAX_ROW_HEADS / 4, table_width < 1 or a scale that is not finite. Lengths beyond 2^30 are taken as 2^30. */
size_t knnssd_paged_attention_bytes(const knnssd_pages *pages, int32_t n_heads, int32_t dtype);
int32_t knnssd_paged_attention(const knnssd_pages *pages, const int32_t *block_table_dev, int32_t table_width,
                               const int32_t *row_start_dev, const int32_t *kv_len_dev, int32_t n_requests,
                               const void *q_dev, int64_t q_stride, void *out_dev, int64_t out_stride, int32_t dtype, int32_t n_rows,
                               int32_t n_heads, float scale, int32_t most_rows, void *ws_dev, size_t ws_bytes, void *hip_stream);

/* Attention of whole prompts, each over itself, causal: rows row_start[r] .. row_start[r+1]-1 are request r's positions 0, 1, ... q, k, v and
 * out are rows of n_heads (q, out) or n_kv_heads (k, v) heads of head_dim values in dtype, their strides in elements; q, k and v may be parts of
 * the same rows; k_stride and v_stride at most 2^26 (KNNSSD_ESHAPE). Otherwise as knnssd_paged_attention; no pages, no workspace. */
int32_t knnssd_prompt_attention(const void *q_dev, int64_t q_stride, const void *k_dev, int64_t k_stride, const void *v_dev,
                                int64_t v_stride, void *out_dev, int64_t out_stride, int32_t dtype, const int32_t *row_start_dev,
                                int32_t n_requests, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                                void *hip_stream);

/* One block of a context's own cache as pages of page_size positions (page g: positions g*page_size ...), so that the calls above read what
 * knnssd_prefill, knnssd_draft_step and knnssd_verify have written. Host only. KNNSSD_ERANGE for a block outside the model, KNNSSD_ESHAPE if max_seq
 * is not a multiple of page_size or page_size is not one that knnssd_pages allows. */
int32_t knnssd_context_pages(const knnssd_ctx *ctx, int32_t block, int32_t page_size, knnssd_pages *pages_out);

/* ---- Trees of drafted tokens ------------------------------------------------------------------------------------
 * A batch's new rows may be trees of drafted tokens instead of chains: parents[t] says for row t of the batch which row of its request (0: the request's first) it continues; -1, or
 * anything that is not an earlier row, makes it a root. Row 0 is the last token that is certain, the others are drafts. A round: knnssd_page_plan, knnssd_tree_plan, for every block
 * knnssd_paged_store (with the tree's positions) and knnssd_tree_attention, then knnssd_tree_verify and knnssd_tree_keep, whose lengths are the next plan's `cached`.
 * What is said above of batches holds here too: everything in stream order, capturable, lengths and trees read on the device and bounded there.           */
#define KNNSSD_MAX_TREE 1024                /* rows of a request's tree */
#define KNNSSD_MAX_VOCAB (1 << 19)

/* Positions and masks of ancestors. positions_dev [n_rows]: kv_len[r] minus the request's rows plus the row's depth (a root's is 0), over those that knnssd_page_plan wrote (a row's slot stays: the
 * tree's rows lie in the cache in their own order). masks_dev [n_rows][mask_words], 8-byte aligned: bit j % 64 of word j / 64 says that the row sees row j of its request: itself and its ancestors. A
 * request has up to 64 * mask_words rows; the masks of further ones are 0 and their positions -1. Rows behind the last request's are left as they were. row_start_dev and kv_len_dev as
 * knnssd_page_plan wrote them. Outputs must not overlap inputs or each other (KNNSSD_EINVAL). KNNSSD_ERANGE for mask_words outside [1, KNNSSD_MAX_TREE / 64], n_requests outside [1, KNNSSD_MAX_REQUESTS], n_rows outside [1, KNNSSD_MAX_ROW_HEADS / 4]. */
int32_t knnssd_tree_plan(const int32_t *parents_dev, const int32_t *row_start_dev, const int32_t *kv_len_dev, int32_t n_requests, int32_t n_rows,
                         int32_t *positions_dev, uint64_t *masks_dev, int32_t mask_words, void *hip_stream);

/* knnssd_paged_attention for rows that see, of their request's new rows, only those up to themselves whose bits in their masks are set (any mask will do: row i sees row j <= i if bit j is set, rows
 * from 64 * mask_words on have no bit), and all cached positions. A row that sees nothing has an output of 0. Workspace and limits as there; keys and values of
 * all of a request's new rows have to be finite. masks_dev: [n_rows][mask_words], 8-byte aligned. */
int32_t knnssd_tree_attention(const knnssd_pages *pages, const int32_t *block_table_dev, int32_t table_width, const int32_t *row_start_dev,
                              const int32_t *kv_len_dev, int32_t n_requests, const uint64_t *masks_dev, int32_t mask_words, const void *q_dev, int64_t q_stride,
                              void *out_dev, int64_t out_stride, int32_t dtype, int32_t n_rows, int32_t n_heads, float scale, int32_t most_rows,
                              void *ws_dev, size_t ws_bytes, void *hip_stream);

/* Drafted tokens tried against the model's probabilities, so that what comes out is distributed as the model's own tokens are. logits_dev: [n_rows] rows of vocab values in dtype, logits_stride
 * elements apart (any alignment of the type's own), -inf for tokens that are ruled out; row t's are those of the token behind row t. p = softmax(logits / temperature[r]); at a temperature of 0
 * all of it is on the (first) largest value. From row 0 on the children of the node reached so far are tried in the order of their rows, with the row's number u from u_accept_dev [n_rows]:
 *   draft_logits_dev given (rows as logits'; a row's are those that its children were drawn from, each for itself, with the same temperature; rows without children are not looked at):
 *     q = softmax(draft_logits / temperature); c = 0, S = 1 at first; child x is taken if p(x) > (c + u S) q(x), else, if q(x) > 0, c grows by S and S becomes the sum of max(p - c q, 0)
 *   draft_logits_dev NULL, the drafts were not drawn: child x is taken if p(x) > u S, else S loses p(x) and p(x) becomes 0
 * Where no child is taken the walk ends, and the next token is the first that the sum of max(p - c q, 0) (or of what is left of p) up to and with it is more than u_next[r] times the whole sum. So a
 * request of a single row draws a token from its logits. A request's path_dev[row_start[r] + j], j < n_path[r], are its rows taken, row 0 first, -1 behind; next_token_dev[r] comes
 * behind them. All sums are in 64 bits, of exponentials that are off by up to 2.2e-12 of them; in the sums of max(p - c q, 0) and where the next token is picked, values of p (and of q) that are 2^-500 of their row's
 * largest and less count as nothing, so that such a token is not the next one under a u_next of 0 either. Numbers from [0, 1) belong in u_accept_dev and u_next_dev.
 * next_token[r] is -1 where there is no distribution to go by: a request without rows or with a temperature that is negative or not finite (n_path is 0 then), a row on the path whose logits (or, if it has
 * children, draft's logits) hold NaN or +inf or nothing but -inf, or nothing left of p (S of given drafts is
 * 1 less what was tried, in 64 bits: where they are all of p's tokens and all but 10^-12 of it has been rejected, the last one may be too). A drafted token outside the vocabulary is never taken; rows from
 * KNNSSD_MAX_TREE on of a request are none of the tree. most_children: an upper bound of a row's children if the caller has one, else 0; it only chooses the kernels.
 * ws_dev: knnssd_tree_verify_bytes (drawn: draft_logits_dev is given; 0: sizes that the call refuses), 256-byte aligned, of any contents; nothing in it outlives a call. The same call gives the same result.
 * KNNSSD_ESHAPE for vocab outside [1, KNNSSD_MAX_VOCAB], KNNSSD_ERANGE for n_requests outside [1, KNNSSD_MAX_REQUESTS], n_rows outside [1, KNNSSD_MAX_ROW_HEADS / 4] or
 * n_rows * ceil(vocab / 2048) > KNNSSD_MAX_ROW_HEADS. Outputs must not overlap the int32 and float inputs or each other
 * (KNNSSD_EINVAL), nor what else is read. */
size_t knnssd_tree_verify_bytes(int32_t n_rows, int32_t n_requests, int32_t vocab, int32_t drawn);
int32_t knnssd_tree_verify(const void *logits_dev, int64_t logits_stride, const void *draft_logits_dev, int64_t draft_stride, int32_t dtype, int32_t vocab,
                           const int32_t *tokens_dev, const int32_t *parents_dev, const int32_t *row_start_dev, int32_t n_requests, int32_t n_rows,
                           const float *temperature_dev, const float *u_accept_dev, const float *u_next_dev, int32_t *path_dev, int32_t *n_path_dev,
                           int32_t *next_token_dev, int32_t most_children, void *ws_dev, size_t ws_bytes, void *hip_stream);

/* The path's keys and values side by side: in every one of n_blocks caches (alike in everything but their addresses: KNNSSD_ESHAPE) the entry of row path[row_start[r] + j] of request r goes to position
 * kv_len[r] - rows + j, for j < n_path[r]; cached_dev[r] becomes the position behind the last of them, the next knnssd_page_plan's `cached`. A path ascends strictly; it ends before an entry that does
 * not, that is no row of the request or that lies beyond its table. What a request's positions from cached[r] on hold afterwards is of no use. cached_dev must not overlap an input, and no cache be given twice, as keys
 * and values of one block or in two blocks that share one (KNNSSD_EINVAL). KNNSSD_ERANGE for n_blocks outside [1, 1024], table_width < 1, n_requests or n_rows as in knnssd_tree_plan. */
int32_t knnssd_tree_keep(const knnssd_pages *blocks, int32_t n_blocks, const int32_t *block_table_dev, int32_t table_width, const int32_t *row_start_dev,
                         const int32_t *kv_len_dev, int32_t n_requests, int32_t n_rows, const int32_t *path_dev, const int32_t *n_path_dev,
                         int32_t *cached_dev, void *hip_stream);

/* Message for an error code; for KNNSSD_EHIP the text of the last HIP error of this thread. */
const char *knnssd_strerror(int32_t code);

#ifdef __cplusplus
}
#endif
#endif /* KNNSSD_H */
