// Host-side checks of what the batch calls are given.
#pragma once
#include <stdint.h>

#include "../../include/knnssd.h"

static inline bool page_size_ok(int32_t p) { return p >= 8 && p <= 1024 && (p & (p - 1)) == 0; }

static inline bool dtype_ok(int32_t t) { return t == KNNSSD_FP32 || t == KNNSSD_BF16; }

static inline int64_t dtype_bytes(int32_t t) { return t == KNNSSD_BF16 ? 2 : 4; }

// rows (or pages) read and written in 16-byte pieces: the base, and a stride of at least `least` elements
static inline bool rows_ok(const void *base, int64_t stride, int64_t least, int32_t dtype) {
    return !((uintptr_t)base & 15) && stride >= least && stride <= INT64_MAX / 8 && !((stride * dtype_bytes(dtype)) & 15);
}

// distance of neighbouring positions (or rows of keys), which the kernels count in 32 bits of bytes over a few of them
static const int64_t MAX_ROW_STRIDE = 1 << 26;

// KNNSSD_OK, or what is wrong with a paged cache
static inline int32_t pages_check(const knnssd_pages *p) {
    if (!p || !p->k_dev || !p->v_dev) return KNNSSD_EINVAL;
    if (!dtype_ok(p->kv_dtype)) return KNNSSD_EINVAL;
    if ((p->head_dim != 64 && p->head_dim != 128) || p->n_kv_heads < 1 || p->n_kv_heads > 65535) return KNNSSD_ESHAPE;
    if (!page_size_ok(p->page_size) || p->n_pages < 1 || (int64_t)p->n_pages * p->page_size > INT32_MAX) return KNNSSD_ESHAPE;
    if (!rows_ok(p->k_dev, p->pos_stride, p->head_dim, p->kv_dtype) || !rows_ok(p->v_dev, p->head_stride, p->head_dim, p->kv_dtype) ||
        !rows_ok(p->k_dev, p->page_stride, p->head_dim, p->kv_dtype))
        return KNNSSD_EINVAL;
    return p->pos_stride > MAX_ROW_STRIDE ? KNNSSD_ESHAPE : KNNSSD_OK;
}

// words of a row's mask in a tree
static inline bool mask_words_ok(int32_t words) { return words >= 1 && words <= KNNSSD_MAX_TREE / 64; }

// the types that rows and a cache may have together
static inline bool types_go_together(int32_t rows, int32_t cache) { return rows == KNNSSD_FP32 || cache == KNNSSD_BF16; }
