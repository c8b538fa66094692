// Attention of a batch's rows in fp32: over pages (PAGED) or over their own prompts' rows.
#pragma once
#include "battn_common.h"

namespace ks {

// A wavefront per (row, head), fp32: the lanes that share a position take eight dimensions each, 64 / (HD / 8) positions at a time;
// each such group of lanes keeps its own running maximum and sum, merged at the end.
template <int HD, bool PAGED>
__global__ __launch_bounds__(256) void battn_row_kernel(BattnArgs a) {
    constexpr int LP = HD / 8, NP = 64 / LP;
    const int lane = threadIdx.x & 63;
    const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(item / a.H), h = (int)(item % a.H), kvh = h / a.group;
    if (t >= a.n_rows || t >= a.row_start[a.n_requests]) return;
    const int r = battn_request(a.row_start, a.n_requests, t), r0 = max(a.row_start[r], 0);
    const int n = a.row_start[r + 1] - r0;
    const int len = PAGED ? battn_len(a, r) : n;
    const int last = PAGED ? min(len - n + (t - r0), len - 1) : t - r0;      // the row's own position
    const int d = (lane % LP) * 8, sub = lane / LP;
    float q[8], o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float *qp = (const float *)a.q + t * a.q_stride + h * HD + d;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = qp[e];
    float m = -INFINITY, l = 0.f;
    for (int p = sub; p <= last; p += NP) {
        long long ko, vo;
        if constexpr (PAGED) {
            ko = vo = battn_paged(a, r, kvh, p);
        } else {
            ko = (long long)(r0 + p) * a.k_stride + kvh * HD;
            vo = (long long)(r0 + p) * a.v_stride + kvh * HD;
        }
        const float *kp = (const float *)a.k + ko + d, *vp = (const float *)a.v + vo + d;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(q[e], kp[e], s);
        for (int off = 1; off < LP; off <<= 1) s += __shfl_xor(s, off);
        s *= a.scale2;
        const float mn = fmaxf(m, s), f = exp2f(m - mn), w = exp2f(s - mn);
        l = l * f + w;
        m = mn;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(w, vp[e], o[e] * f);
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
        store_values<8>((float *)a.out + t * a.out_stride + h * HD + d, o);
    }
}

}  // namespace ks
