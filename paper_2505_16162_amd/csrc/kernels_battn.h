// Attention of a batch's rows over pages (PAGED) or over their own prompts' rows.
#pragma once
#include "kernels_pages.h"

namespace ks {

struct BattnArgs {
    const void *q, *k, *v;
    void *out;
    long long q_stride, out_stride;             // rows of q and out
    long long k_stride, v_stride;               // rows of k and v (prompts)
    long long page_stride, head_stride, pos_stride;
    const int *table, *row_start, *kv_len;      // (kv_len, table: pages)
    int n_requests, n_rows, width, shift, n_pages;
    int H, Hkv, group;
    float scale2;                               // scale * log2(e): softmax in powers of two
};

// request of row t < row_start[n], by bisection
__device__ __forceinline__ int battn_request(const int *row_start, int n, int t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// element where position p of request r begins for kv head h. A page id outside the cache reads page 0 instead.
__device__ __forceinline__ long long battn_paged(const BattnArgs &a, int r, int h, int p) {
    const int g = a.table[(size_t)r * a.width + (p >> a.shift)];
    return ((unsigned)g < (unsigned)a.n_pages ? g : 0) * a.page_stride + h * a.head_stride + (p & ((1 << a.shift) - 1)) * a.pos_stride;
}

// A wavefront per (row, head), for any types: the lanes that share a position take eight dimensions each, 64 / (HD / 8) positions at a time;
// each such group of lanes keeps its own running maximum and sum, merged at the end.
template <int HD, bool PAGED, typename T, typename KT>
__global__ __launch_bounds__(256) void battn_row_kernel(BattnArgs a) {
    constexpr int LP = HD / 8, NP = 64 / LP;
    const int lane = threadIdx.x & 63;
    const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(item / a.H), h = (int)(item % a.H), kvh = h / a.group;
    if (t >= a.n_rows || t >= a.row_start[a.n_requests]) return;
    const int r = battn_request(a.row_start, a.n_requests, t), r0 = max(a.row_start[r], 0);
    const int n = a.row_start[r + 1] - r0;
    const int len = PAGED ? (int)min((long long)a.kv_len[r], (long long)a.width << a.shift) : n;
    const int last = PAGED ? min(len - n + (t - r0), len - 1) : t - r0;      // the row's own position
    const int d = (lane % LP) * 8, sub = lane / LP;
    float q[8], o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T *qp = (const T *)a.q + t * a.q_stride + h * HD + d;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = load_as_float(qp, e);
    float m = -INFINITY, l = 0.f;
    for (int p = sub; p <= last; p += NP) {
        long long ko, vo;
        if constexpr (PAGED) {
            ko = vo = battn_paged(a, r, kvh, p);
        } else {
            ko = (long long)(r0 + p) * a.k_stride + kvh * HD;
            vo = (long long)(r0 + p) * a.v_stride + kvh * HD;
        }
        const KT *kp = (const KT *)a.k + ko + d, *vp = (const KT *)a.v + vo + d;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(q[e], load_as_float(kp, e), s);
        for (int off = 1; off < LP; off <<= 1) s += __shfl_xor(s, off);
        s *= a.scale2;
        const float mn = fmaxf(m, s), f = exp2f(m - mn), w = exp2f(s - mn);
        l = l * f + w;
        m = mn;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(w, load_as_float(vp, e), o[e] * f);
    }
    for (int off = LP; off < 64; off <<= 1) {
        const float m2 = __shfl_xor(m, off), l2 = __shfl_xor(l, off), mn = fmaxf(m, m2);
        const float f = m == -INFINITY ? 0.f : exp2f(m - mn), f2 = m2 == -INFINITY ? 0.f : exp2f(m2 - mn);
        l = l * f + l2 * f2;
        m = mn;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * f + __shfl_xor(o[e], off) * f2;
    }
    if (sub == 0) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
        store_values<8>((T *)a.out + t * a.out_stride + h * HD + d, o);
    }
}

}  // namespace ks
