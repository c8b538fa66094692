// Host side of the calls for trees of drafted tokens: plan, verification, keeping a path. (Attention: knnssd_batch.hip.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <functional>

#include "hip_try.h"
#include "kernels_tree.h"
#include "kernels_tverify.h"
#include "pages_check.h"

using namespace ks;

static const int KEEP_MOST_BLOCKS = 1024;                     // what a cache that is given twice is looked for among

static const_ints ints(const int32_t *p) { return (const_ints)(uintptr_t)p; }

// what every call on a batch's rows is given
static int32_t batch_check(const int32_t *row_start_dev, int32_t n_requests, int32_t n_rows) {
    if (!row_start_dev) return KNNSSD_EINVAL;
    return n_requests < 1 || n_requests > KNNSSD_MAX_REQUESTS || n_rows < 1 || n_rows > KNNSSD_MAX_ROW_HEADS / 4 ? KNNSSD_ERANGE : KNNSSD_OK;
}

// Whether an output has entries of an input (or another output): workgroups of other requests would read them before or after.
struct Ints { const void *at; int64_t n; int bytes = 4; };
static bool overlap(const Ints &a, const Ints &b) {
    const uintptr_t x = (uintptr_t)a.at, y = (uintptr_t)b.at;
    return x < y + (uintptr_t)(b.n * b.bytes) && y < x + (uintptr_t)(a.n * a.bytes);
}
template <int OUT, int IN> static bool overlap(const Ints (&out)[OUT], const Ints (&in)[IN]) {
    for (int o = 0; o < OUT; ++o) {
        for (const Ints &i : in)
            if (overlap(out[o], i)) return true;
        for (int x = 0; x < o; ++x)
            if (overlap(out[o], out[x])) return true;
    }
    return false;
}

extern "C" int32_t knnssd_tree_plan(const int32_t *parents_dev, const int32_t *row_start_dev, const int32_t *kv_len_dev, int32_t n_requests, int32_t n_rows,
                                    int32_t *positions_dev, uint64_t *masks_dev, int32_t mask_words, void *hip_stream) {
    if (!parents_dev || !kv_len_dev || !positions_dev || !masks_dev || ((uintptr_t)masks_dev & 7)) return KNNSSD_EINVAL;
    KS_TRY(batch_check(row_start_dev, n_requests, n_rows));
    if (!mask_words_ok(mask_words)) return KNNSSD_ERANGE;
    const Ints out[] = {{positions_dev, n_rows}, {masks_dev, (int64_t)n_rows * mask_words, 8}}, in[] = {{parents_dev, n_rows}, {row_start_dev, n_requests + 1}, {kv_len_dev, n_requests}};
    if (overlap(out, in)) return KNNSSD_EINVAL;
    TreePlanArgs a{};
    a.parents = parents_dev; a.row_start = ints(row_start_dev); a.kv_len = ints(kv_len_dev); a.masks = (unsigned long long *)masks_dev; a.positions = positions_dev;
    a.n_rows = n_rows; a.words = mask_words;
    hipLaunchKernelGGL(tree_plan_kernel, dim3(n_requests), dim3(64 * mask_words), 0, (hipStream_t)hip_stream, a);
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}

static int tv_chunks(int32_t vocab) { return (vocab + TV_CHUNK - 1) / TV_CHUNK; }

// where in the workspace what lies
struct TvLayout { size_t nodes, states, sums, total; };
static TvLayout tv_layout(int64_t n_rows, int64_t n_requests, int32_t vocab, bool drawn) {
    TvLayout l{};
    l.nodes = (size_t)n_rows * tv_chunks(vocab) * sizeof(TvStat) * (drawn ? 2 : 1);
    l.states = l.nodes + (drawn ? n_rows * sizeof(TvNode) : 0);
    l.sums = l.states + (drawn ? n_requests * sizeof(TvState) : 0);
    l.total = (l.sums + (drawn ? n_requests * tv_chunks(vocab) * sizeof(double) : 0) + 255) / 256 * 256;
    return l;
}

static int32_t tv_sizes_check(int32_t n_rows, int32_t n_requests, int32_t vocab) {
    if (n_requests < 1 || n_requests > KNNSSD_MAX_REQUESTS || n_rows < 1 || n_rows > KNNSSD_MAX_ROW_HEADS / 4) return KNNSSD_ERANGE;
    if (vocab < 1 || vocab > KNNSSD_MAX_VOCAB) return KNNSSD_ESHAPE;
    return (int64_t)n_rows * tv_chunks(vocab) > KNNSSD_MAX_ROW_HEADS ? KNNSSD_ERANGE : KNNSSD_OK;
}

extern "C" size_t knnssd_tree_verify_bytes(int32_t n_rows, int32_t n_requests, int32_t vocab, int32_t drawn) {
    return tv_sizes_check(n_rows, n_requests, vocab) == KNNSSD_OK ? tv_layout(n_rows, n_requests, vocab, drawn != 0).total : 0;
}

static bool values_ok(const void *base, int64_t stride, int32_t vocab, int32_t dtype) {
    return !((uintptr_t)base & (dtype_bytes(dtype) - 1)) && stride >= vocab && stride <= INT64_MAX / 8;
}

// How many sums over a row are taken by launches of their own, spread over the chip, before a walk's workgroup takes those that are still needed by itself. A round costs 4 us where no walk waits and
// about 12 where one does, a sum by one workgroup 0.6 us for every 2048 tokens. Whole calls of 12 requests, us, with 0, 1, 2, 3, 4 rounds:
//   trees of 8 to 40 rows, 4096 tokens 20, 28, 35, 39, 42; 16384 36, 39, 41, 44, 47; 32000 65, 61, 55, 56, 57; 64000 119, 101, 87, 75, 70; 152064 (6 to 20 rows) 211, 156, 96, 78, 82
//   chains of 1 to 9 rows, 8192 tokens 19, 25, 28, 31, 40; 32000 35, 29, 32, 35, 39; 152064 102, 42, 44, 47, 50
static int verify_rounds(int chunks, int most_children) { return chunks <= 8 ? 0 : most_children == 1 ? 1 : chunks <= 24 ? 2 : 4; }

// Whether the rows' sums are taken by a table of powers (bf16): where there are enough chunks for a table in every compute unit, and for each request's. Whole calls, us, without / with:
//   256 requests of 4 rows of 50000 (25 600 chunks) 46 / 36; 16 of 24 of 152064 (28 800) 52 / 42; 256 of 1 of 152064 (19 200) 36 / 29; 1 of 120 of 152064 (9000) 34 / 33; 128 of 2 of 64000
//   (8192, 64 a request) 24.2 / 24.1; 64 of 1 of 152064 (4800) 21.2 / 21.8; 512 of 1 of 32000 (8192, 16 a request) 23 / 26.5; drawn chains of 9 rows, 256 of 152064 535 / 365, 64 of 64000 74 / 68
// Where it has nothing to give it costs: all greedy (16 of 24) 27 / 31; a logit of exactly 0 in every chunk 52 / 68.
static bool by_table(const TvArgs &a, unsigned units) { return units >= 8192 && units / 64 >= (unsigned)a.n_requests; }

template <typename T>
static void launch_verify(const TvArgs &a, int rounds, hipStream_t s) {
    const unsigned units = (unsigned)a.n_rows * a.chunks * (a.draft ? 2 : 1);
    if (sizeof(T) == 2 && by_table(a, units)) hipLaunchKernelGGL(tv_stats_table_kernel, dim3(TT_WGS), dim3(TT_NT), 0, s, a);
    else hipLaunchKernelGGL((tv_stats_kernel<T>), dim3((units + 3) / 4), dim3(256), 0, s, a);
    for (int i = 0; i <= rounds; ++i) {
        if (i > 0) hipLaunchKernelGGL((tv_sum_kernel<T>), dim3(a.chunks, a.n_requests), dim3(256), 0, s, a);
        hipLaunchKernelGGL((tv_walk_kernel<T>), dim3(a.n_requests), dim3(TV_NT), 0, s, a, i, i < rounds);
    }
}

extern "C" int32_t knnssd_tree_verify(const void *logits_dev, int64_t logits_stride, const void *draft_logits_dev, int64_t draft_stride, int32_t dtype, int32_t vocab,
                                      const int32_t *tokens_dev, const int32_t *parents_dev, const int32_t *row_start_dev, int32_t n_requests, int32_t n_rows,
                                      const float *temperature_dev, const float *u_accept_dev, const float *u_next_dev, int32_t *path_dev, int32_t *n_path_dev,
                                      int32_t *next_token_dev, int32_t most_children, void *ws_dev, size_t ws_bytes, void *hip_stream) {
    if (!logits_dev || !tokens_dev || !parents_dev || !row_start_dev || !temperature_dev || !u_accept_dev || !u_next_dev) return KNNSSD_EINVAL;
    if (!path_dev || !n_path_dev || !next_token_dev || !ws_dev || !dtype_ok(dtype)) return KNNSSD_EINVAL;
    KS_TRY(tv_sizes_check(n_rows, n_requests, vocab));
    if (most_children < 0) return KNNSSD_ERANGE;
    if (!values_ok(logits_dev, logits_stride, vocab, dtype) || (draft_logits_dev && !values_ok(draft_logits_dev, draft_stride, vocab, dtype))) return KNNSSD_EINVAL;
    if (((uintptr_t)ws_dev & 255) || ws_bytes < knnssd_tree_verify_bytes(n_rows, n_requests, vocab, draft_logits_dev != nullptr)) return KNNSSD_EINVAL;
    const Ints out[] = {{path_dev, n_rows}, {n_path_dev, n_requests}, {next_token_dev, n_requests}};
    const Ints in[] = {{tokens_dev, n_rows}, {parents_dev, n_rows}, {row_start_dev, n_requests + 1}, {temperature_dev, n_requests}, {u_accept_dev, n_rows}, {u_next_dev, n_requests}};
    if (overlap(out, in)) return KNNSSD_EINVAL;
    const TvLayout l = tv_layout(n_rows, n_requests, vocab, draft_logits_dev != nullptr);
    TvArgs a{};
    a.logits = logits_dev; a.draft = draft_logits_dev; a.logits_stride = logits_stride; a.draft_stride = draft_stride;
    a.tokens = tokens_dev; a.parents = parents_dev; a.row_start = ints(row_start_dev);
    a.temperature = temperature_dev; a.u_accept = u_accept_dev; a.u_next = u_next_dev;
    a.path = path_dev; a.n_path = n_path_dev; a.next = next_token_dev;
    a.stats = (TvStat *)ws_dev; a.nodes = (TvNode *)((char *)ws_dev + l.nodes); a.states = (TvState *)((char *)ws_dev + l.states); a.sums = (double *)((char *)ws_dev + l.sums);
    a.n_requests = n_requests; a.n_rows = n_rows; a.vocab = vocab; a.chunks = tv_chunks(vocab);
    const int rounds = draft_logits_dev ? verify_rounds(a.chunks, most_children) : 0;        // (only then the workspace has room for walks between rounds)
    if (dtype == KNNSSD_BF16) launch_verify<bf16_t>(a, rounds, (hipStream_t)hip_stream);
    else launch_verify<float>(a, rounds, (hipStream_t)hip_stream);
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}

extern "C" int32_t knnssd_tree_keep(const knnssd_pages *blocks, int32_t n_blocks, const int32_t *block_table_dev, int32_t table_width, const int32_t *row_start_dev,
                                    const int32_t *kv_len_dev, int32_t n_requests, int32_t n_rows, const int32_t *path_dev, const int32_t *n_path_dev,
                                    int32_t *cached_dev, void *hip_stream) {
    if (!blocks || !block_table_dev || !kv_len_dev || !path_dev || !n_path_dev || !cached_dev) return KNNSSD_EINVAL;
    KS_TRY(batch_check(row_start_dev, n_requests, n_rows));
    if (n_blocks < 1 || n_blocks > KEEP_MOST_BLOCKS || table_width < 1) return KNNSSD_ERANGE;
    const knnssd_pages &p = blocks[0];
    for (int i = 0; i < n_blocks; ++i) {
        const knnssd_pages &o = blocks[i];
        KS_TRY(pages_check(&o));
        if (o.page_stride != p.page_stride || o.head_stride != p.head_stride || o.pos_stride != p.pos_stride || o.n_pages != p.n_pages || o.page_size != p.page_size ||
            o.n_kv_heads != p.n_kv_heads || o.head_dim != p.head_dim || o.kv_dtype != p.kv_dtype)
            return KNNSSD_ESHAPE;
    }
    // (the workgroups of other blocks read a request's lengths when the first one may have written what is left of them)
    const Ints out[] = {{cached_dev, n_requests}};
    const Ints in[] = {{kv_len_dev, n_requests}, {n_path_dev, n_requests}, {row_start_dev, n_requests + 1}, {path_dev, n_rows}, {block_table_dev, (int64_t)n_requests * table_width}};
    if (overlap(out, in)) return KNNSSD_EINVAL;
    // (a cache that is given twice, as keys and values of one block or as two blocks that share theirs, would be moved twice, the second time what has been moved)
    const void *bases[2 * KEEP_MOST_BLOCKS];
    for (int i = 0; i < n_blocks; ++i) { bases[2 * i] = blocks[i].k_dev; bases[2 * i + 1] = blocks[i].v_dev; }
    std::sort(bases, bases + 2 * n_blocks, std::less<const void *>());
    if (std::adjacent_find(bases, bases + 2 * n_blocks) != bases + 2 * n_blocks) return KNNSSD_EINVAL;
    const int64_t elt = dtype_bytes(p.kv_dtype);
    TreeKeepArgs a{};
    a.page_stride = p.page_stride * elt; a.head_stride = p.head_stride * elt; a.pos_stride = p.pos_stride * elt;
    a.table = ints(block_table_dev); a.row_start = ints(row_start_dev); a.kv_len = ints(kv_len_dev); a.path = ints(path_dev); a.n_path = ints(n_path_dev);
    a.n_rows = n_rows; a.width = table_width; a.shift = __builtin_ctz((unsigned)p.page_size); a.n_pages = p.n_pages;
    a.head_pieces = (int)(p.head_dim * elt / 16);
    a.pieces = p.n_kv_heads * a.head_pieces;
    for (int b0 = 0; b0 < n_blocks; b0 += KEEP_BLOCKS) {
        const int n = n_blocks - b0 < KEEP_BLOCKS ? n_blocks - b0 : KEEP_BLOCKS;
        for (int i = 0; i < n; ++i) { a.k[i] = blocks[b0 + i].k_dev; a.v[i] = blocks[b0 + i].v_dev; }
        a.cached = b0 == 0 ? cached_dev : nullptr;
        hipLaunchKernelGGL(tree_keep_kernel, dim3(n_requests, n, (2 * a.pieces + KEEP_NT - 1) / KEEP_NT), dim3(KEEP_NT), 0, (hipStream_t)hip_stream, a);
    }
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}
