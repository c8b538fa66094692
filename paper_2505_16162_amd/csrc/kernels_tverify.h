// Drafted tokens tried against the target's probabilities.
#pragma once
#include <cfloat>

#include "../../include/knnssd.h"
#include "device_ops.h"
#include "rows_range.h"

namespace ks {

// ------------------------------------------------------------------------------------------
// p = softmax(logits / T) of a node's row, q the same of the draft's logits there. Children of a node are tried in the order of their rows. Drawn from q, the distribution that is
// left after j of them were rejected is max(p - c q, 0) / S, with c = 0, S = 1 before the first and c += S, S = sum max(p - c q, 0) behind each: rejecting a draw from q takes S q off
// S times that distribution. So child x passes if u < max(p(x) - c q(x), 0) / (S q(x)), that is p(x) > (c + u S) q(x). Drafts that were not drawn (the most likely tokens, say) are
// draws from a distribution that is all on x: x passes if p(x) > u S, else S -= p(x) and p(x) = 0.
// All of it in 64 bits: of 150 000 tokens' cumulative sums neighbours are nearer to each other than sums of fp32 exponentials are to the right ones, and the wrong neighbour is the wrong token.
//
// tv_stats_kernel: largest value and sum of exponentials of every 2048 values of every row, a wavefront each, so that any row spreads over the chip. It reads the logits
// once and is bound by memory and by the exponentials beside it, 19 instructions in 64 bits a value.
// tv_walk_kernel: a workgroup per request puts rows together, gets all drafted tokens' probabilities at once, walks, and picks the next token.
// tv_sum_kernel: S behind a rejection, spread over the chip.
// ------------------------------------------------------------------------------------------
constexpr int TV_CHUNK = 2048;                                // values of a wavefront
constexpr int TV_NT = 1024, TV_WAVES = TV_NT / 64;            // the walk's threads

struct TvStat { float top; int first; double sum; };          // largest value, its first place (temperature 0), sum of 2^((value - top) k); NaN: the row has no distribution

// weights of a row's tokens: max(p - c q, 0), p = p_each 2^((value - p_top) k), c q = q_each 2^((value - q_top) k); or those of p alone
struct TvWeigh { float p_top, q_top; double p_each, q_each, k; };

// a walk between two rounds: waits for the sums of w's weights over the row of `node`
struct TvState {
    TvWeigh w;
    double c;
    int node, last, kept, waits;
};

struct TvArgs {
    const void *logits, *draft;                               // draft: NULL if the drafts were not drawn
    long long logits_stride, draft_stride;
    const int *tokens, *parents;
    const_ints row_start;
    const float *temperature, *u_accept, *u_next;
    int *path, *n_path, *next;
    TvStat *stats;                                            // [rows][chunks], behind them the same of the draft
    TvState *states;                                          // [requests] (drawn)
    double *sums;                                             // [requests][chunks] (drawn)
    int n_requests, n_rows, vocab, chunks;
};

// 2^x for x <= 0: 2^n 2^r with |r| <= 1/2, 2^r by its Taylor polynomial of degree 10 (what is cut off: 2e-13 of it). Below 2^-1100 (NaN too): 0.
__device__ __forceinline__ double tv_exp2(double x) {
    x = __builtin_fmax(x, -1100.0);
    const double n = __builtin_rint(x), r = x - n;
    double p = 7.0549116208011233e-09;                        // ln(2)^i / i!
    p = __builtin_fma(p, r, 1.0178086009239700e-07);
    p = __builtin_fma(p, r, 1.3215486790144309e-06);
    p = __builtin_fma(p, r, 1.5252733804059840e-05);
    p = __builtin_fma(p, r, 1.5403530393381609e-04);
    p = __builtin_fma(p, r, 1.3333558146428443e-03);
    p = __builtin_fma(p, r, 9.6181291076284772e-03);
    p = __builtin_fma(p, r, 5.5504108664821580e-02);
    p = __builtin_fma(p, r, 2.4022650695910071e-01);
    p = __builtin_fma(p, r, 6.9314718055994531e-01);
    p = __builtin_fma(p, r, 1.0);
    return __builtin_ldexp(p, (int)n);
}

// eight values of a row from `at` on, -inf behind its last
typedef unsigned int tv_words __attribute__((ext_vector_type(4)));
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) TvPiece { tv_words w; };      // (rows begin anywhere)
__device__ __forceinline__ void tv_load8(const float *row, int at, int vocab, float *v) {
    if (at + 8 <= vocab) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const tv_words w = reinterpret_cast<const TvPiece<float> *>(row + at + 4 * h)->w;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * h + e] = __uint_as_float(w[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = at + e < vocab ? row[at + e] : -INFINITY;
    }
}
__device__ __forceinline__ void tv_load8(const bf16_t *row, int at, int vocab, float *v) {
    if (at + 8 <= vocab) {
        const tv_words w = reinterpret_cast<const TvPiece<bf16_t> *>(row + at)->w;
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(w[e] << 16); v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = at + e < vocab ? bf16_to_float(row[at + e]) : -INFINITY;
    }
}
// where the lane's i-th eight of a chunk begin
__device__ __forceinline__ int tv_at(int chunk, int i, int lane) { return chunk * TV_CHUNK + (i * 64 + lane) * 8; }

__device__ __forceinline__ double tv_sum(double v, int width = 64) {
    for (int off = width >> 1; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}
__device__ __forceinline__ float tv_max(float v, int width) {
    for (int off = width >> 1; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void tv_stats_kernel(TvArgs a) {
    const int lane = threadIdx.x & 63;
    int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const bool draft = unit >= a.n_rows * a.chunks;
    if (draft) unit -= a.n_rows * a.chunks;
    const int row = unit / a.chunks, chunk = unit - row * a.chunks;
    if (row >= a.n_rows || (draft && !a.draft)) return;                              // (from here on wavefronts are on their own)
    const int r = battn_request(a.row_start, a.n_requests, row);
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int i = row - rows.first;
    if (i < 0 || i >= rows.n || i >= KNNSSD_MAX_TREE) return;
    if (draft) {                                              // a row without children: its draft's logits are nobody's
        bool child = false;
        for (int j = i + 1 + lane; j < min(rows.n, KNNSSD_MAX_TREE); j += 64) child = child || a.parents[rows.first + j] == i;
        if (!__any(child)) return;
    }
    const T *from = (const T *)(draft ? a.draft : a.logits) + row * (draft ? a.draft_stride : a.logits_stride);
    float v[4][8];
#pragma unroll
    for (int q = 0; q < 4; ++q) tv_load8(from, tv_at(chunk, q, lane), a.vocab, v[q]);
    const float t = a.temperature[r];
    float top = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            top = fmaxf(top, v[q][e]);
            bad = bad || !(v[q][e] <= FLT_MAX);
        }
    top = wave_max(top);
    bad = __any(bad);
    double sum = 0.0;
    int first = INT32_MAX;
    if (t > 0.f && top > -INFINITY) {
        const double k = 1.4426950408889634 / (double)t, m = top;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += tv_exp2(((double)v[q][e] - m) * k);
        sum = tv_sum(sum);
    } else {
#pragma unroll
        for (int q = 3; q >= 0; --q)
#pragma unroll
            for (int e = 7; e >= 0; --e)
                if (v[q][e] == top) first = tv_at(chunk, q, lane) + e;
        for (int off = 32; off > 0; off >>= 1) first = min(first, __shfl_xor(first, off));
    }
    if (lane == 0) a.stats[(size_t)(draft ? a.n_rows : 0) * a.chunks + unit] = TvStat{top, first, bad ? (double)NAN : sum};
}

// What a walk knows of a node's row: largest value and sum, or (temperature 0) the first place of the largest value. `top` is NaN if the row has no distribution.
struct TvRow { float top; int first; double sum; };

// lanes of a group of `width` put a row's chunks together
__device__ __forceinline__ TvRow tv_join(const TvStat *s, int chunks, double k, int in, int width) {
    TvRow row{-INFINITY, INT32_MAX, 0.0};
    for (int c = in; c < chunks; c += width) row.top = fmaxf(row.top, s[c].top);
    row.top = tv_max(row.top, width);
    for (int c = in; c < chunks; c += width) {
        const TvStat one = s[c];
        if (one.top > -INFINITY) row.sum += one.sum * tv_exp2(((double)one.top - row.top) * k);
        else if (one.sum != one.sum) row.sum = one.sum;
        if (one.top == row.top) row.first = min(row.first, one.first);
    }
    row.sum = tv_sum(row.sum, width);
    for (int off = width >> 1; off > 0; off >>= 1) row.first = min(row.first, __shfl_xor(row.first, off));
    if (row.sum != row.sum || row.top == -INFINITY) row.top = NAN;
    return row;
}

// ... of a lane's eight tokens
template <typename T>
__device__ __forceinline__ void tv_weights(const TvWeigh &w, const T *p, const T *q, int at, int vocab, double *out) {
    float v[8];
    tv_load8(p, at, vocab, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = w.p_each * tv_exp2(((double)v[e] - (double)w.p_top) * w.k);
    if (q) {
        tv_load8(q, at, vocab, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = __builtin_fmax(__builtin_fma(-w.q_each, tv_exp2(((double)v[e] - (double)w.q_top) * w.k), out[e]), 0.0);
    }
}
// ... without the tokens that were rejected
__device__ __forceinline__ void tv_without(const int *rejected, int n, int at, double *w) {
    for (int x = 0; x < n; ++x) {
        const int d = rejected[x] - at;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d == e) w[e] = 0.0;
    }
}

// sum of a chunk's weights, the same in all lanes
template <typename T>
__device__ __forceinline__ double tv_chunk_sum(const TvWeigh &w, const T *p, const T *q, int chunk, int lane, int vocab, const int *rejected, int n_rejected) {
    double sum = 0.0;
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        double v[8];
        const int at = tv_at(chunk, i, lane);
        tv_weights(w, p, q, at, vocab, v);
        tv_without(rejected, n_rejected, at, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e];
    }
    return tv_sum(sum);
}

// The chunk's first token that the weights up to and with it are more than `target`, or (roundings) its last one with a weight; -1 without any.
template <typename T>
__device__ __forceinline__ int tv_pick(const TvWeigh &w, const T *p, const T *q, int chunk, int lane, int vocab, const int *rejected, int n_rejected, double target) {
    double before = 0.0;
    int best = -1;                                            // the lane's last token with a weight
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        double v[8], mine = 0.0;
        const int at = tv_at(chunk, i, lane);
        tv_weights(w, p, q, at, vocab, v);
        tv_without(rejected, n_rejected, at, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mine += v[e];
            if (v[e] > 0.0) best = at + e;
        }
        double upto = mine;
        for (int off = 1; off < 64; off <<= 1) {
            const double x = __shfl_up(upto, off);
            if (lane >= off) upto += x;
        }
        double run = before + (upto - mine);
        int found = INT32_MAX;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            run += v[e];
            if (found == INT32_MAX && v[e] > 0.0 && run > target) found = at + e;
        }
        for (int off = 32; off > 0; off >>= 1) found = min(found, __shfl_xor(found, off));
        if (found != INT32_MAX) return found;
        before += __shfl(upto, 63);
    }
    for (int off = 32; off > 0; off >>= 1) best = max(best, __shfl_xor(best, off));
    return best;
}

// Rounds: a rejected draw needs the sum over its whole row before the walk can go on. One compute unit takes 40 us for rows of 150 000 tokens, so the walk of `round` stops
// there if a launch of tv_sum_kernel and another round follow (`more`), and goes on in that; a walk that has no further round takes the sums that it still needs by itself.
template <typename T>
__global__ __launch_bounds__(TV_NT) void tv_walk_kernel(TvArgs a, int round, int more) {
    __shared__ int parent[KNNSSD_MAX_TREE], token[KNNSSD_MAX_TREE], u_bits[KNNSSD_MAX_TREE];
    __shared__ TvRow p_row[KNNSSD_MAX_TREE], q_row[KNNSSD_MAX_TREE];
    __shared__ double p_at[KNNSSD_MAX_TREE], q_at[KNNSSD_MAX_TREE], chunk_sum[KNNSSD_MAX_VOCAB / TV_CHUNK];
    __shared__ bool inner[KNNSSD_MAX_TREE];                   // has children
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int n = min(rows.n, KNNSSD_MAX_TREE);
    const float t = a.temperature[r];
    const bool drawn = a.draft != nullptr, greedy = t == 0.f;
    const double k = greedy ? 0.0 : 1.4426950408889634 / (double)t;
    TvState s{};
    if (round > 0) {
        s = a.states[r];
        if (!s.waits) return;
    } else if (n == 0 || !(t >= 0.f && t <= FLT_MAX)) {
        for (int i = tid; i < rows.n; i += TV_NT) a.path[rows.first + i] = -1;
        if (tid == 0) {
            a.n_path[r] = 0;
            a.next[r] = -1;
            if (more) a.states[r].waits = 0;
        }
        return;
    }
    for (int i = tid; i < n; i += TV_NT) {
        const int p = a.parents[rows.first + i], x = a.tokens[rows.first + i];
        parent[i] = p >= 0 && p < i && (unsigned)x < (unsigned)a.vocab ? p : -1;        // (a token that is none never passes)
        token[i] = x;
        u_bits[i] = __float_as_int(a.u_accept[rows.first + i]);
        inner[i] = false;
    }
    __syncthreads();
    for (int i = tid; i < n; i += TV_NT)
        if (parent[i] >= 0) inner[parent[i]] = true;
    if (round == 0)
        for (int i = tid; i < rows.n; i += TV_NT) a.path[rows.first + i] = i == 0 ? 0 : -1;
    __syncthreads();
    // the rows' sums put together, a group of lanes each; the draft's where it has been asked for any
    const TvStat *p_stats = a.stats + (size_t)rows.first * a.chunks, *q_stats = p_stats + (size_t)a.n_rows * a.chunks;
    int width = 1;
    while (width < a.chunks && width < 64) width <<= 1;
    const int in = tid & (width - 1);
    for (int i = tid / width; i < n; i += TV_NT / width) {
        const TvRow p = tv_join(p_stats + (size_t)i * a.chunks, a.chunks, k, in, width);
        if (in == 0) p_row[i] = p;
        if (drawn && inner[i]) {
            const TvRow q = tv_join(q_stats + (size_t)i * a.chunks, a.chunks, k, in, width);
            if (in == 0) q_row[i] = q;
        }
    }
    __syncthreads();
    // every drafted token's probabilities at its parent
    const T *logits = (const T *)a.logits + rows.first * a.logits_stride, *draft = (const T *)a.draft + (drawn ? rows.first * a.draft_stride : 0);
    for (int i = tid; i < n; i += TV_NT) {
        const int p = parent[i], x = token[i];
        if (p < 0) continue;
        auto at = [&](const T *row, const TvRow &of) { return greedy ? (x == of.first ? 1.0 : 0.0) : tv_exp2(((double)load_as_float(row, x) - of.top) * k) / of.sum; };
        p_at[i] = at(logits + p * a.logits_stride, p_row[p]);
        if (drawn) q_at[i] = at(draft + p * a.draft_stride, q_row[p]);
    }
    __syncthreads();

    // the walk, the same in all wavefronts: `node`, its child `last` that was tried last, and what of p is left
    int node = 0, last = 0, kept = 1;
    double c = 0.0, left = 1.0;
    bool summed = false, lost = false;                        // chunk_sum has the node's weights; a row without a distribution
    auto add_up = [&]() {                                     // ... of all chunks
        __syncthreads();
        double total = 0.0;
        for (int x = lane; x < a.chunks; x += 64) total += chunk_sum[x];
        return tv_sum(total);
    };
    if (round > 0) {
        node = s.node; last = s.last; kept = s.kept; c = s.c;
        for (int x = tid; x < a.chunks; x += TV_NT) chunk_sum[x] = a.sums[(size_t)r * a.chunks + x];
        left = add_up();
        summed = true;
    }
    while (true) {
        if (p_row[node].top != p_row[node].top || (drawn && inner[node] && q_row[node].top != q_row[node].top)) {
            lost = true;
            break;
        }
        int child = -1;
        for (int i0 = (last + 1) & ~63; i0 < n && child < 0 && inner[node]; i0 += 64) {
            const int i = i0 + lane;
            const unsigned long long found = __ballot(i < n && i > last && parent[i] == node);
            if (found) child = i0 + __builtin_ctzll(found);
        }
        if (child < 0) break;
        last = child;
        const double u = __int_as_float(u_bits[child]);
        double px = p_at[child];
        if (!drawn) {                                         // the same token again: it has been rejected
            for (int i0 = (node + 1) & ~63; i0 < child; i0 += 64) {
                const int i = i0 + lane;
                if (__any(i < child && i > node && parent[i] == node && token[i] == token[child])) px = 0.0;
            }
        }
        const double qx = drawn ? q_at[child] : 1.0;
        if (px > (c + u * left) * qx) {
            node = child;
            if (tid == 0) a.path[rows.first + kept] = child;
            ++kept;
            c = 0.0;
            left = 1.0;
            summed = false;
        } else if (!drawn) {
            left -= px;
        } else if (qx > 0.0) {                                // (a token that the draft cannot have drawn says nothing about its distribution)
            c += left;
            if (greedy) {
                left = 1.0;                                   // (p and q are each all on one token, not the same: p stays)
                continue;
            }
            const TvWeigh w{p_row[node].top, q_row[node].top, 1.0 / p_row[node].sum, c / q_row[node].sum, k};
            if (more) {
                if (tid == 0) {
                    a.states[r] = TvState{w, c, node, last, kept, 1};
                    a.n_path[r] = kept;
                }
                return;
            }
            __syncthreads();                                  // (the last sums have been read)
            for (int x = wave; x < a.chunks; x += TV_WAVES) {
                const double sum = tv_chunk_sum(w, logits + node * a.logits_stride, draft + node * a.draft_stride, x, lane, a.vocab, nullptr, 0);
                if (lane == 0) chunk_sum[x] = sum;
            }
            left = add_up();
            summed = true;
        }
    }
    if (tid == 0) {
        a.n_path[r] = kept;
        if (more) a.states[r].waits = 0;
        if (lost || greedy) a.next[r] = lost ? -1 : p_row[node].first;
    }
    if (lost || greedy) return;

    // the next token: of max(p - c q, 0), or of p without the rejected tokens
    __shared__ int n_rejected;
    int *rejected = u_bits;
    __syncthreads();                                          // (the numbers have been read)
    if (tid == 0) n_rejected = 0;
    __syncthreads();
    const T *p = logits + node * a.logits_stride, *q = summed ? draft + node * a.draft_stride : nullptr;
    const TvWeigh w{p_row[node].top, summed ? q_row[node].top : 0.f, summed ? 1.0 / p_row[node].sum : 1.0, summed ? c / q_row[node].sum : 0.0, k};
    if (!drawn) {
        for (int i = tid; i < n; i += TV_NT)
            if (parent[i] == node) rejected[atomicAdd(&n_rejected, 1)] = token[i];       // (in any order: all of them get a weight of 0)
        __syncthreads();
    }
    const int gone = n_rejected;
    if (!summed) {
        const TvStat *own = p_stats + (size_t)node * a.chunks;
        for (int x = wave; x < a.chunks; x += TV_WAVES) {
            bool again = false;                               // a rejected token lies here
            for (int i = lane; i < gone; i += 64) again = again || rejected[i] / TV_CHUNK == x;
            double sum;
            if (__any(again)) sum = tv_chunk_sum(w, p, q, x, lane, a.vocab, rejected, gone);
            else sum = own[x].top > -INFINITY ? own[x].sum * tv_exp2(((double)own[x].top - w.p_top) * k) : 0.0;
            if (lane == 0) chunk_sum[x] = sum;
        }
    }
    const double total = add_up();
    if (wave != 0) return;
    const double target = (double)a.u_next[r] * total;
    int chunk = -1, holds = -1;                               // the chunk that the target lies in; the last one with a weight
    double before = 0.0, chunk_before = 0.0, holds_before = 0.0;
    for (int x0 = 0; x0 < a.chunks && chunk < 0; x0 += 64) {
        const double mine = x0 + lane < a.chunks ? chunk_sum[x0 + lane] : 0.0;
        double upto = mine;
        for (int off = 1; off < 64; off <<= 1) {
            const double x = __shfl_up(upto, off);
            if (lane >= off) upto += x;
        }
        const unsigned long long any = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && before + upto > target);
        const double here = before + (upto - mine);
        if (past) {
            const int l = __builtin_ctzll(past);
            chunk = x0 + l;
            chunk_before = __shfl(here, l);
        } else if (any) {
            const int l = 63 - __builtin_clzll(any);
            holds = x0 + l;
            holds_before = __shfl(here, l);
        }
        before += __shfl(upto, 63);
    }
    if (chunk < 0) {
        chunk = holds;
        chunk_before = holds_before;
    }
    int next = -1;
    if (chunk >= 0) next = tv_pick(w, p, q, chunk, lane, a.vocab, rejected, gone, target - chunk_before);
    if (lane == 0) a.next[r] = next;
}

// Sums of max(p - c q, 0) over the chunks of the rows at which walks wait, a wavefront each.
template <typename T>
__global__ __launch_bounds__(256) void tv_sum_kernel(TvArgs a) {
    const int r = blockIdx.y, chunk = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (chunk >= a.chunks || !a.states[r].waits) return;
    const TvState s = a.states[r];
    const long long row = rows_of(a.row_start, r, a.n_rows).first + s.node;
    const double sum = tv_chunk_sum(s.w, (const T *)a.logits + row * a.logits_stride, (const T *)a.draft + row * a.draft_stride, chunk, lane, a.vocab, nullptr, 0);
    if (lane == 0) a.sums[(size_t)r * a.chunks + chunk] = sum;
}

}  // namespace ks
