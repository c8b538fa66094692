// Host side of the batch calls of the C ABI: page plans, rotary store into pages, attention over pages and over prompts.
#include <hip/hip_runtime.h>

#include <cmath>

#include "hip_try.h"
#include "kernels_battn_few.h"
#include "kernels_battn_row.h"
#include "kernels_battn_tile.h"
#include "kernels_pages.h"
#include "pages_check.h"

using namespace ks;

static int log2_of(int v) { return __builtin_ctz((unsigned)v); }

extern "C" int32_t knnssd_page_plan(const knnssd_page_tables *t, const int32_t *cached_dev, const int32_t *added_dev,
                                    const knnssd_batch_rows *rows, void *hip_stream) {
    if (!t || !rows || !cached_dev || !added_dev) return KNNSSD_EINVAL;
    if (!t->block_table_dev || !t->held_dev || !t->free_pages_dev || !t->n_free_dev) return KNNSSD_EINVAL;
    if (!rows->row_start_dev || !rows->kv_len_dev || !rows->slots_dev || !rows->positions_dev || !rows->result_dev) return KNNSSD_EINVAL;
    if (t->n_requests < 1 || t->n_requests > KNNSSD_MAX_REQUESTS || rows->max_rows < 1) return KNNSSD_ERANGE;
    if (!page_size_ok(t->page_size) || t->n_pages < 1 || (int64_t)t->n_pages * t->page_size > INT32_MAX) return KNNSSD_ESHAPE;
    if (t->table_width < 1 || (int64_t)t->n_requests * t->table_width > INT32_MAX) return KNNSSD_ESHAPE;
    PlanArgs a{};
    a.table = t->block_table_dev; a.held = t->held_dev; a.free_pages = t->free_pages_dev; a.n_free = t->n_free_dev;
    a.cached = cached_dev; a.added = added_dev;
    a.row_start = rows->row_start_dev; a.kv_len = rows->kv_len_dev; a.slots = rows->slots_dev; a.positions = rows->positions_dev; a.result = rows->result_dev;
    a.n = t->n_requests; a.width = t->table_width; a.n_pages = t->n_pages; a.shift = log2_of(t->page_size); a.max_rows = rows->max_rows;
    a.rows_here = rows->max_rows <= 2048;
    hipStream_t s = (hipStream_t)hip_stream;
    // Few wavefronts meet sooner (48 requests: 5.4 us, with 1024 threads 8.6), many move pages faster (256 prompts admitted, 12 000 pages: 15 us, with 256 threads 36).
    // No more pages change hands than the table has entries.
    if (a.n <= 256 && a.rows_here && (int64_t)a.n * a.width <= 8192) hipLaunchKernelGGL((page_plan_kernel<256, 1>), dim3(1), dim3(256), 0, s, a);
    else if (a.n <= 1024) hipLaunchKernelGGL((page_plan_kernel<1024, 1>), dim3(1), dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((page_plan_kernel<1024, 4>), dim3(1), dim3(1024), 0, s, a);
    if (!a.rows_here) {
        const int wgs = (int)(((int64_t)rows->max_rows + PLAN_ROWS_NT - 1) / PLAN_ROWS_NT);
        hipLaunchKernelGGL(page_rows_kernel, dim3(wgs < 1024 ? wgs : 1024), dim3(PLAN_ROWS_NT), 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}

template <int HD>
static void launch_store(const StoreArgs &a, int32_t dtype, int32_t kv_dtype, int n_rows, hipStream_t s) {
    const int per = HD / 2 / (dtype == KNNSSD_BF16 ? 8 : 4), items = (a.n_heads + 2 * a.n_kv) * per;
    const dim3 grid(n_rows, (items + STORE_NT * STORE_U - 1) / (STORE_NT * STORE_U));
    if (dtype == KNNSSD_BF16) hipLaunchKernelGGL((paged_store_kernel<HD, bf16_t, bf16_t>), grid, dim3(STORE_NT), 0, s, a);
    else if (kv_dtype == KNNSSD_BF16) hipLaunchKernelGGL((paged_store_kernel<HD, float, bf16_t>), grid, dim3(STORE_NT), 0, s, a);
    else hipLaunchKernelGGL((paged_store_kernel<HD, float, float>), grid, dim3(STORE_NT), 0, s, a);
}

extern "C" int32_t knnssd_paged_store(const knnssd_pages *p, const void *qkv_dev, int32_t dtype, int64_t qkv_stride, int32_t n_rows,
                                      int32_t n_heads, const int32_t *slots_dev, const int32_t *positions_dev, float rope_base,
                                      void *q_out_dev, int64_t q_out_stride, void *k_out_dev, int64_t k_out_stride, void *hip_stream) {
    KS_TRY(pages_check(p));
    if (!qkv_dev || !slots_dev || !positions_dev) return KNNSSD_EINVAL;
    if (!dtype_ok(dtype) || !types_go_together(dtype, p->kv_dtype)) return KNNSSD_EINVAL;
    if (n_rows < 1 || n_rows > KNNSSD_MAX_ROW_HEADS / 4 || n_heads < 0 || n_heads > 65535 || !(rope_base > 0.f) || !std::isfinite(rope_base)) return KNNSSD_ERANGE;
    const int64_t hd = p->head_dim;
    if (!rows_ok(qkv_dev, qkv_stride, (n_heads + 2 * (int64_t)p->n_kv_heads) * hd, dtype)) return KNNSSD_EINVAL;
    if (q_out_dev && !rows_ok(q_out_dev, q_out_stride, n_heads * hd, dtype)) return KNNSSD_EINVAL;
    if (k_out_dev && !rows_ok(k_out_dev, k_out_stride, p->n_kv_heads * hd, dtype)) return KNNSSD_EINVAL;
    StoreArgs a{};
    a.qkv = qkv_dev; a.q_out = q_out_dev; a.k_out = k_out_dev; a.k = p->k_dev; a.v = p->v_dev; a.slots = slots_dev; a.positions = positions_dev;
    a.qkv_stride = qkv_stride; a.q_stride = q_out_stride; a.k_stride = k_out_stride;
    a.page_stride = p->page_stride; a.head_stride = p->head_stride; a.pos_stride = p->pos_stride;
    a.n_heads = n_heads; a.n_kv = p->n_kv_heads; a.shift = log2_of(p->page_size); a.n_slots = p->n_pages * p->page_size;
    a.log2_base = std::log2((double)rope_base);
    if (hd == 128) launch_store<128>(a, dtype, p->kv_dtype, n_rows, (hipStream_t)hip_stream);
    else launch_store<64>(a, dtype, p->kv_dtype, n_rows, (hipStream_t)hip_stream);
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}

// what both attention calls are given: a batch's rows of q and out
static int32_t rows_check(const int32_t *row_start_dev, int32_t n_requests, const void *q, int64_t q_stride, const void *out, int64_t out_stride,
                          int32_t dtype, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int64_t hd, float scale) {
    if (!row_start_dev || !q || !out || !dtype_ok(dtype)) return KNNSSD_EINVAL;
    if (n_requests < 1 || n_requests > KNNSSD_MAX_REQUESTS || n_rows < 1 || !std::isfinite(scale)) return KNNSSD_ERANGE;
    if (n_heads < 1 || n_heads > 65535 || n_heads % n_kv_heads) return KNNSSD_ESHAPE;
    if ((int64_t)n_rows * n_heads > KNNSSD_MAX_ROW_HEADS || (int64_t)n_requests * n_heads > KNNSSD_MAX_ROW_HEADS / 4) return KNNSSD_ERANGE;
    if (!rows_ok(q, q_stride, n_heads * hd, dtype) || !rows_ok(out, out_stride, n_heads * hd, dtype)) return KNNSSD_EINVAL;
    return KNNSSD_OK;
}

template <int HD, int NP>
static void launch_merge(const BattnArgs &a, unsigned runs, int pairs, int64_t groups, int slot_pairs, hipStream_t s) {
    // few groups lie in many runs each, whose pairs then take four teams of lanes
    const int at_once = groups < BF_WGS / 4 ? battn_merge_teams<HD>() / 4 : battn_merge_teams<HD>();
    hipLaunchKernelGGL((battn_merge_kernel<HD, NP>), dim3(runs, (pairs + at_once - 1) / at_once), dim3(BM_NT), 0, s, a, slot_pairs);
}

// tiles at most; what is too much ends at once
static int64_t tiles_bound(const BattnArgs &a) { return (((int64_t)a.n_rows * a.group + BT_PAIRS - 1) / BT_PAIRS + a.n_requests) * a.Hkv; }

template <int HD, int NP>
static void launch_paged_tiles(const BattnArgs &a, int64_t most, hipStream_t s) {
    hipLaunchKernelGGL((battn_tile_kernel<HD, true, NP>), dim3(BF_WGS), dim3(256), (battn_tile_lds<HD, true, NP>()), s, a);
    launch_merge<HD, NP == 1 ? 1 : 3>(a, BF_WGS, (int)(most < BT_PAIRS ? most : BT_PAIRS), tiles_bound(a), BT_PAIRS, s);
}

template <int HD, int NP>
static void launch_prompt_tiles(const BattnArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((battn_tile_kernel<HD, false, NP>), dim3((unsigned)tiles_bound(a)), dim3(256), (battn_tile_lds<HD, false, NP>()), s, a);
}

// Most (row, head) pairs of one kv head that a request may have for battn_few_kernel to take the batch: as many as one group holds; each further group reads the cache
// again. Whole calls, us, few rows / tiles, 32 requests at 200 to 4000 positions, bf16 queries; fp32 ones (whose tiles do three times the products):
//   40 heads of 128 over 8: 5 pairs 62 / 68; 59 / 83, 10 to 15 64 / 72; 67 / 91, 20 77 / 57; 104 / 88, 20 to 30 92 / 63; 85 / 78, 35 to 60 133 / 64; 189 / 118
//   40 over 40: 1 pair 233 / 271; 240 / 296, 16 293 / 306; 286 / 339, 20 527 / 319; 557 / 404, 60 972 / 384; 1011 / 433
//   32 heads of 64 over 8: 8 to 12 29 / 31; 34 / 52, 16 34 / 39; 40 / 54, 16 to 24 42 / 38; 51 / 57, 28 to 48 58 / 37; 70 / 64
// Two requests of 20 to 30 pairs at 100 000 positions 223 / 157; 227 / 167. The bound is the caller's most_rows, or all rows of the batch.
static const int FEW_PAIRS = 16;

template <int HD, int NP>
static void launch_few(const BattnArgs &a, int64_t most, hipStream_t s) {
    const int ch = battn_few_positions<HD>();
    const int64_t blocks = (((int64_t)a.width << a.shift) + ch - 1) / ch, groups = ((int64_t)a.n_rows * a.group + FEW_PAIRS - 1) / (FEW_PAIRS) + a.n_requests;
    const int64_t units = blocks < INT32_MAX ? blocks * groups * a.Hkv : INT64_MAX;      // at most
    const unsigned runs = (unsigned)(units / 4 + 1 < BF_WGS ? (units / 4 + 8) & -8 : BF_WGS);
    hipLaunchKernelGGL((battn_few_kernel<HD, NP>), dim3(runs), dim3(256), 0, s, a);
    launch_merge<HD, NP>(a, runs, (int)(most < FEW_PAIRS ? most : FEW_PAIRS), groups * a.Hkv, FEW_PAIRS, s);
}

// In fp32 the tiles' matrix instructions take 8000 cycles a block, however few pairs a tile has; few rows over short contexts are done sooner by battn_row_kernel.
// What the host knows of a context's length is the most that its table holds, so the same requests go to the tiles under a table for more. Whole calls, us, row kernel / tiles:
// three prompts of 45 rows, 4 heads of 64, 8 / 15; one row of 40 heads of 128 over 400 positions 11 / 22, eight requests of one 26 / 29; 32 requests of one row,
// 4 heads of 64, 8 / 27. It loses where many heads of one kv head read the same keys: 32 requests of one row, 40 heads over 8, 400 positions 101 / 44 (100 positions 28 / 28).
static bool rows_alone(const BattnArgs &a, int64_t positions) { return (int64_t)a.n_rows * a.H < BR_FULL && positions <= 512; }

template <int HD>
static void launch_paged(const BattnArgs &a, int32_t dtype, int32_t kv_dtype, int32_t most_rows, hipStream_t s) {
    const int64_t most = (int64_t)(most_rows > 0 && most_rows < a.n_rows ? most_rows : a.n_rows) * a.group;
    if (kv_dtype == KNNSSD_FP32) {
        if (rows_alone(a, (int64_t)a.width << a.shift)) hipLaunchKernelGGL((battn_row_kernel<HD, true>), dim3((unsigned)(a.n_rows * a.H)), dim3(256), 0, s, a);
        else launch_paged_tiles<HD, 0>(a, most, s);
    } else if (most <= FEW_PAIRS) {
        if (dtype == KNNSSD_FP32) launch_few<HD, 3>(a, most, s);
        else launch_few<HD, 1>(a, most, s);
    } else {
        if (dtype == KNNSSD_FP32) launch_paged_tiles<HD, 3>(a, most, s);
        else launch_paged_tiles<HD, 1>(a, most, s);
    }
}

template <int HD>
static void launch_prompts(const BattnArgs &a, int32_t dtype, hipStream_t s) {
    if (dtype == KNNSSD_BF16) launch_prompt_tiles<HD, 1>(a, s);
    else if (rows_alone(a, a.n_rows)) hipLaunchKernelGGL((battn_row_kernel<HD, false>), dim3((unsigned)(a.n_rows * a.H)), dim3(256), 0, s, a);
    else launch_prompt_tiles<HD, 0>(a, s);
}

extern "C" size_t knnssd_paged_attention_bytes(const knnssd_pages *p, int32_t n_heads, int32_t dtype) {
    if (pages_check(p) != KNNSSD_OK || !dtype_ok(dtype) || !types_go_together(dtype, p->kv_dtype)) return 0;
    if (n_heads < 1 || n_heads > 65535 || n_heads % p->n_kv_heads) return 0;
    const size_t slot = p->head_dim == 128 ? battn_few_slot<128>(BT_PAIRS) : battn_few_slot<64>(BT_PAIRS);
    return battn_few_merges() + 2 * BF_WGS * slot * sizeof(float);
}

extern "C" int32_t knnssd_paged_attention(const knnssd_pages *p, const int32_t *block_table_dev, int32_t table_width,
                                          const int32_t *row_start_dev, const int32_t *kv_len_dev, int32_t n_requests, const void *q_dev,
                                          int64_t q_stride, void *out_dev, int64_t out_stride, int32_t dtype, int32_t n_rows, int32_t n_heads,
                                          float scale, int32_t most_rows, void *ws_dev, size_t ws_bytes, void *hip_stream) {
    KS_TRY(pages_check(p));
    if (!block_table_dev || !kv_len_dev || !ws_dev) return KNNSSD_EINVAL;
    KS_TRY(rows_check(row_start_dev, n_requests, q_dev, q_stride, out_dev, out_stride, dtype, n_rows, n_heads, p->n_kv_heads, p->head_dim, scale));
    if (!types_go_together(dtype, p->kv_dtype)) return KNNSSD_EINVAL;
    if (table_width < 1 || most_rows < 0) return KNNSSD_ERANGE;
    if (((uintptr_t)ws_dev & 255) || ws_bytes < knnssd_paged_attention_bytes(p, n_heads, dtype)) return KNNSSD_EINVAL;
    BattnArgs a{};
    a.q = q_dev; a.k = p->k_dev; a.v = p->v_dev; a.out = out_dev; a.q_stride = q_stride; a.out_stride = out_stride;
    a.page_stride = p->page_stride; a.head_stride = p->head_stride; a.pos_stride = p->pos_stride;
    a.table = (const_ints)(uintptr_t)block_table_dev; a.row_start = (const_ints)(uintptr_t)row_start_dev; a.kv_len = (const_ints)(uintptr_t)kv_len_dev;
    a.n_requests = n_requests; a.n_rows = n_rows; a.width = table_width; a.shift = log2_of(p->page_size); a.n_pages = p->n_pages;
    a.H = n_heads; a.Hkv = p->n_kv_heads; a.group = n_heads / p->n_kv_heads;
    a.scale2 = scale * 1.4426950408889634f;
    a.ws = ws_dev;
    if (p->head_dim == 128) launch_paged<128>(a, dtype, p->kv_dtype, most_rows, (hipStream_t)hip_stream);
    else launch_paged<64>(a, dtype, p->kv_dtype, most_rows, (hipStream_t)hip_stream);
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}

extern "C" int32_t knnssd_prompt_attention(const void *q_dev, int64_t q_stride, const void *k_dev, int64_t k_stride, const void *v_dev,
                                           int64_t v_stride, void *out_dev, int64_t out_stride, int32_t dtype, const int32_t *row_start_dev,
                                           int32_t n_requests, int32_t n_rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                           float scale, void *hip_stream) {
    if (!k_dev || !v_dev) return KNNSSD_EINVAL;
    if ((head_dim != 64 && head_dim != 128) || n_kv_heads < 1) return KNNSSD_ESHAPE;
    KS_TRY(rows_check(row_start_dev, n_requests, q_dev, q_stride, out_dev, out_stride, dtype, n_rows, n_heads, n_kv_heads, head_dim, scale));
    if (!rows_ok(k_dev, k_stride, (int64_t)n_kv_heads * head_dim, dtype) || !rows_ok(v_dev, v_stride, (int64_t)n_kv_heads * head_dim, dtype)) return KNNSSD_EINVAL;
    if (k_stride > MAX_ROW_STRIDE || v_stride > MAX_ROW_STRIDE) return KNNSSD_ESHAPE;
    BattnArgs a{};
    a.q = q_dev; a.k = k_dev; a.v = v_dev; a.out = out_dev; a.q_stride = q_stride; a.out_stride = out_stride; a.k_stride = k_stride; a.v_stride = v_stride;
    a.row_start = (const_ints)(uintptr_t)row_start_dev; a.n_requests = n_requests; a.n_rows = n_rows;
    a.H = n_heads; a.Hkv = n_kv_heads; a.group = n_heads / n_kv_heads;
    a.scale2 = scale * 1.4426950408889634f;
    if (head_dim == 128) launch_prompts<128>(a, dtype, (hipStream_t)hip_stream);
    else launch_prompts<64>(a, dtype, (hipStream_t)hip_stream);
    HIP_TRY(hipGetLastError());
    return KNNSSD_OK;
}
