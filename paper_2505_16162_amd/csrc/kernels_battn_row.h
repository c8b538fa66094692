// Attention of a batch's rows in fp32: over pages (PAGED) or over their own prompts' rows.
#pragma once
#include "battn_common.h"

namespace ks {

// A (row, head) at a time, in fp32 from end to end, for the smallest calls: the lanes that share a position take eight dimensions each, 64 / (HD / 8) positions
// at a time, four such steps under way; each such group of lanes keeps its own running maximum and sum, merged at the end, and the four
// wavefronts of a workgroup share the item's positions. Bound by memory latency; keys and values are read once for every row and head, from the caches
// (34 requests of up to 8 rows, 5 heads, 100 to 350 positions: 19 us; with one wavefront and one step at a time 59).
constexpr int BR_FULL = 4096;                                 // (row, head) items from which the tiles are taken instead

// TREE (pages): of the new rows a row sees those that its mask has.
template <int HD, bool PAGED, bool TREE>
__global__ __launch_bounds__(256) void battn_row_kernel(BattnArgs a) {
    constexpr int LP = HD / 8, NP = 64 / LP, U = 4, W = 4;
    __shared__ float part[4][HD + 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = blockIdx.x / a.H, h = blockIdx.x % a.H, kvh = h / a.group;
    if (t >= a.n_rows || t >= a.row_start[a.n_requests]) return;      // the whole workgroup
    const int r = battn_request(a.row_start, a.n_requests, t);
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int r0 = rows.first, n = rows.n;
    const int len = PAGED ? battn_len(a, r) : n;
    const int last = PAGED ? min(len - n + (t - r0), len - 1) : t - r0;      // the row's own position
    BattnMask mask{};
    if constexpr (TREE) mask = battn_mask(a, t);
    const int d = (lane % LP) * 8, sub = lane / LP + wave * NP;
    float q[8], o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const float *qp = (const float *)a.q + t * a.q_stride + h * HD + d;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = qp[e];
    float m = -INFINITY, l = 0.f;
    for (int p0 = sub; p0 <= last; p0 += U * NP * W) {        // (the same for the lanes of a position)
        float k[U][8], v[U][8], s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = min(p0 + u * NP * W, last);
            long long ko, vo;
            if constexpr (PAGED) {
                ko = vo = battn_paged(a, r, kvh, p);
            } else {
                ko = (long long)(r0 + p) * a.k_stride + kvh * HD;
                vo = (long long)(r0 + p) * a.v_stride + kvh * HD;
            }
            const float *kp = (const float *)a.k + ko + d, *vp = (const float *)a.v + vo + d;
            Piece<float>::load(kp, k[u]);
            Piece<float>::load(kp + 4, k[u] + 4);
            Piece<float>::load(vp, v[u]);
            Piece<float>::load(vp + 4, v[u] + 4);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            s[u] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[u] = fmaf(q[e], k[u][e], s[u]);
#pragma unroll
            for (int off = 1; off < LP; off <<= 1) s[u] += lane_xor(s[u], off);
            bool sees = p0 + u * NP * W <= last;
            if constexpr (TREE) {
                const int j = p0 + u * NP * W - (len - n);
                if (j >= 0) sees = sees && (mask.word(j >> 6) >> (j & 63) & 1);
            }
            s[u] = sees ? s[u] * a.scale2 : -INFINITY;
            top = fmaxf(top, s[u]);
        }
        const float ref = top == -INFINITY ? 0.f : top, f = exp2f(m - ref);
        m = top;
        l *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = exp2f(s[u] - ref);
            l += w;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(w, v[u][e], o[e]);
        }
    }
    // (v of a position that is not the row's is that of its last one, with a weight of 0)
#pragma unroll
    for (int off = LP; off < 64; off <<= 1) {
        const float m2 = lane_xor(m, off), l2 = lane_xor(l, off), mn = fmaxf(m, m2);
        const float f = m == -INFINITY ? 0.f : exp2f(m - mn), f2 = m2 == -INFINITY ? 0.f : exp2f(m2 - mn);
        l = l * f + l2 * f2;
        m = mn;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * f + lane_xor(o[e], off) * f2;
    }
    if (lane < LP) {
#pragma unroll
        for (int e = 0; e < 8; ++e) part[wave][d + e] = o[e];
        if (lane == 0) { part[wave][HD] = m; part[wave][HD + 1] = l; }
    }
    __syncthreads();
    if (wave != 0) return;
    m = fmaxf(fmaxf(part[0][HD], part[1][HD]), fmaxf(part[2][HD], part[3][HD]));
    l = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const float f = part[x][HD] == -INFINITY ? 0.f : exp2f(part[x][HD] - m);
        l = fmaf(part[x][HD + 1], f, l);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = fmaf(part[x][d + e], f, o[e]);
    }
    if (lane < LP) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= inv;
        store_values<8>((float *)a.out + t * a.out_stride + h * HD + d, o);
    }
}

}  // namespace ks
