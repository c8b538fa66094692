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
// once; what bounds it are the exponentials: 17 instructions in 64 bits a value, and what a wavefront does besides (whose row it is, sums over its lanes). 284 rows of 152064 values in bf16:
// 33.7 us, 2.6 TB/s (without the exponentials 20.7, without the loads 23.5). (By the table, below: 29.4.)
// tv_stats_table_kernel: the same of large batches in bf16, with a table of the powers in place of the polynomial.
// tv_walk_kernel: a workgroup per request puts rows together, gets all drafted tokens' probabilities at once, walks, and picks the next token.
// tv_sum_kernel: S behind a rejection, spread over the chip.
// Walks take 8 us (one tree of 26 rows, 32000 tokens), a chain of dependent loads and steps.
// ------------------------------------------------------------------------------------------
constexpr int TV_CHUNK = 2048;                                // values of a wavefront
constexpr int TV_MAX_CHUNKS = KNNSSD_MAX_VOCAB / TV_CHUNK;
constexpr int TV_NT = 512, TV_WAVES = TV_NT / 64;             // the walk's threads
constexpr int TV_EACH = KNNSSD_MAX_TREE / TV_NT, TV_PICK = TV_CHUNK / TV_NT;       // rows of a tree, tokens of a chunk to a thread

struct TvStat { float top; int first; double sum; };          // largest value, its first place (temperature 0), sum of 2^((value - top) k); NaN: the row has no distribution

// weights of a row's tokens: max(p - c q, 0), p = p_each 2^((value - p_top) k), c q = q_each 2^((value - q_top) k); or those of p alone
struct TvWeigh { float p_top, q_top, p_least, q_least; double p_each, q_each, k; };      // (values below the least count as nothing)

// What a walk knows of a node's row: largest value and sum, or (temperature 0) the first place of the largest value. `top` is NaN if the row has no distribution.
struct TvRow { float top; int first; double sum; };

// a row of a tree between two rounds
struct TvNode {
    TvRow p, q;
    double p_at, q_at;                                        // its token's probabilities at its parent
    int parent, token, u, inner;
};

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
    TvNode *nodes;                                            // [rows] (drawn)
    double *sums;                                             // [requests][chunks] (drawn)
    int n_requests, n_rows, vocab, chunks;
};

// 2^r for |r| <= 1/2: 1 + r times the polynomial that meets (2^r - 1) / r at the eight Chebyshev points. Off by at most 2.2e-12 of it, and exact at 0. N of them side by side: each is a
// chain of dependent instructions.
constexpr double TV_C9 = 1.325080551750225e-06;
template <int N>
__device__ __forceinline__ void tv_poly(const double *r, double *p, double c9 = TV_C9) {
    constexpr double C[8] = {1.5303700711365693e-05, 1.5403475186530786e-04, 1.3333478473685416e-03, 9.61812913523614e-03,
                             5.5504109063258665e-02, 2.4022650695888503e-01, 6.931471805568324e-01,  1.0};
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = c9;
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = __builtin_fma(p[i], r[i], C[c]);
}
// 2^x for x <= 0, down to 0; of NaN: 0
__device__ __forceinline__ double tv_exp2(double x) {
    x = __builtin_fmax(x, -1100.0);
    const double n = __builtin_rint(x), r = x - n;
    double p;
    tv_poly<1>(&r, &p);
    return __builtin_ldexp(p, (int)n);
}
typedef unsigned int tv_pair __attribute__((ext_vector_type(2)));
// 2^(d k) for -1020 <= d k <= 0, with fewer instructions: adding 1.5 * 2^52 leaves the nearest whole number in the low bits, which go to the exponent as they are
template <int N>
__device__ __forceinline__ void tv_exp2_near(const double *d, double k, double *out) {
    double t[N], r[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = __builtin_fma(d[i], k, 0x1.8p52);
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = __builtin_fma(d[i], k, 0x1.8p52 - t[i]);
    tv_poly<N>(r, out);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        tv_pair p = __builtin_bit_cast(tv_pair, out[i]);
        p[1] += __builtin_bit_cast(tv_pair, t[i])[0] << 20;
        out[i] = __builtin_bit_cast(double, p);
    }
}

// Eight values of a row from `at` on as they lie in memory, -inf behind its last. (Rows begin anywhere.)
typedef unsigned int tv_words __attribute__((ext_vector_type(4)));
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) TvPiece { tv_words w; };
template <typename T> struct TvRaw { tv_words w[sizeof(T) / 2]; };
__device__ __forceinline__ void tv_load8(const float *row, int at, TvRaw<float> &raw) {
#pragma unroll
    for (int h = 0; h < 2; ++h) raw.w[h] = reinterpret_cast<const TvPiece<float> *>(row + at + 4 * h)->w;
}
__device__ __forceinline__ void tv_load8(const bf16_t *row, int at, TvRaw<bf16_t> &raw) { raw.w[0] = reinterpret_cast<const TvPiece<bf16_t> *>(row + at)->w; }
__device__ __forceinline__ void tv_load8_end(const float *row, int at, int vocab, TvRaw<float> &raw) {
#pragma unroll
    for (int e = 0; e < 8; ++e) raw.w[e >> 2][e & 3] = at + e < vocab ? __float_as_uint(row[at + e]) : 0xff800000u;
}
__device__ __forceinline__ void tv_load8_end(const bf16_t *row, int at, int vocab, TvRaw<bf16_t> &raw) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const unsigned int lo = at + e < vocab ? row[at + e] : 0xff80u, hi = at + e + 1 < vocab ? row[at + e + 1] : 0xff80u;
        raw.w[0][e >> 1] = lo | hi << 16;
    }
}
__device__ __forceinline__ void tv_values(const TvRaw<float> &raw, float *v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(raw.w[e >> 2][e & 3]);
}
__device__ __forceinline__ void tv_values(const TvRaw<bf16_t> &raw, float *v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(raw.w[0][e] << 16); v[2 * e + 1] = __uint_as_float(raw.w[0][e] & 0xffff0000u); }
}
// where the lane's i-th eight of a chunk begin
__device__ __forceinline__ int tv_at(int chunk, int i, int lane) { return chunk * TV_CHUNK + (i * 64 + lane) * 8; }
// N of them from the first on. (Only a row's last chunk asks where the row ends: loads under a condition of each lane's own would wait for one another.)
template <typename T, int N>
__device__ __forceinline__ void tv_load(const T *row, int chunk, int first, int lane, int vocab, TvRaw<T> *raw) {
    if ((chunk + 1) * TV_CHUNK <= vocab) {
#pragma unroll
        for (int i = 0; i < N; ++i) tv_load8(row, tv_at(chunk, first + i, lane), raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = tv_at(chunk, first + i, lane);
            if (at + 8 <= vocab) tv_load8(row, at, raw[i]);
            else tv_load8_end(row, at, vocab, raw[i]);
        }
    }
}

__device__ __forceinline__ double tv_lane_xor(double v, int off) {
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned int lo = lane_xor((int)b, off), hi = lane_xor((int)(b >> 32), off);
    return __builtin_bit_cast(double, (long long)((unsigned long long)hi << 32 | lo));
}
// over groups of `width` lanes
__device__ __forceinline__ double tv_sum(double v, int width = 64) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        if (off < width) v += tv_lane_xor(v, off);
    return v;
}
__device__ __forceinline__ float tv_max(float v, int width = 64) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        if (off < width) v = fmaxf(v, lane_xor(v, off));
    return v;
}
__device__ __forceinline__ int tv_min(int v, int width = 64) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        if (off < width) v = min(v, lane_xor(v, off));
    return v;
}
// sum over the lanes up to this one: within rows of 16, then the rows' last lanes to the rows behind them
template <int CTRL, int ROWS> __device__ __forceinline__ double tv_lane_behind(double v) {
    tv_pair b = __builtin_bit_cast(tv_pair, v);
    b[0] = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)b[0], CTRL, ROWS, 0xf, false);
    b[1] = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)b[1], CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(double, b);
}
__device__ __forceinline__ double tv_upto(double v) {
    v += tv_lane_behind<0x111, 0xf>(v);                       // row_shr 1, 2, 4, 8
    v += tv_lane_behind<0x112, 0xf>(v);
    v += tv_lane_behind<0x114, 0xf>(v);
    v += tv_lane_behind<0x118, 0xf>(v);
    v += tv_lane_behind<0x142, 0xa>(v);                       // row_bcast 15, 31
    v += tv_lane_behind<0x143, 0xc>(v);
    return v;
}
// lane i's value
__device__ __forceinline__ double tv_lane(double v, int i) {
    const tv_pair b = __builtin_bit_cast(tv_pair, v);
    return __builtin_bit_cast(double, tv_pair{(unsigned int)__builtin_amdgcn_readlane((int)b[0], i), (unsigned int)__builtin_amdgcn_readlane((int)b[1], i)});
}

template <int CTRL, int ROWS> __device__ __forceinline__ float tv_max_behind(float v) {
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xf, false)));
}
// over a wavefront, the same way
__device__ __forceinline__ float tv_max_all(float v) {
    v = tv_max_behind<0x111, 0xf>(v);
    v = tv_max_behind<0x112, 0xf>(v);
    v = tv_max_behind<0x114, 0xf>(v);
    v = tv_max_behind<0x118, 0xf>(v);
    v = tv_max_behind<0x142, 0xa>(v);
    v = tv_max_behind<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Values below this are 2^-500 and less of the largest one: they count as nothing. (Half of what tv_exp2_near allows: the border is rounded to fp32, by
// less than its distance from the top.)
__device__ __forceinline__ float tv_least(float top, float t) { return fmaxf((float)((double)top - 346.5 * t), -FLT_MAX); }      // (500 ln 2)

// (a number for NaN too; fmaxf would take an instruction more)
__device__ __forceinline__ float tv_at_least(float v, float least) { return __builtin_amdgcn_fmed3f(v, least, FLT_MAX); }

// the largest of raw values as signed and as unsigned numbers, in the place of fp32 bits
struct TvBits { int top; unsigned int low; };
__device__ __forceinline__ TvBits tv_bits(const TvRaw<float> *raw) {
    TvBits b{INT32_MIN, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            b.top = max(b.top, (int)raw[q].w[e >> 2][e & 3]);
            b.low = max(b.low, raw[q].w[e >> 2][e & 3]);
        }
    return b;
}
typedef short tv_shorts __attribute__((ext_vector_type(2)));
typedef unsigned short tv_ushorts __attribute__((ext_vector_type(2)));
__device__ __forceinline__ TvBits tv_bits(const TvRaw<bf16_t> *raw) {
    tv_shorts top = {INT16_MIN, INT16_MIN};
    tv_ushorts low = {0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned int two = raw[q].w[0][e];          // (a value of its own: a bit_cast of a vector's element takes the first one)
            top = __builtin_elementwise_max(top, __builtin_bit_cast(tv_shorts, two));
            low = __builtin_elementwise_max(low, __builtin_bit_cast(tv_ushorts, two));
        }
    return TvBits{max(top[0], top[1]) << 16, (unsigned int)max(low[0], low[1]) << 16};
}

// The table of powers 2^(v k) in LDS: entry 2 x + (v < 0) for the x-th |v| from 2^-17 on, x = 1 .. TT_LAST - 1. What is smaller finds NaN (and 0 does), also what is larger and powers beyond
// 2^1000; -inf, and what is below -2^8 or 2^-1000, counts as nothing.
constexpr int TT_LOW = (127 - 17) << 7, TT_LAST = ((127 + 8) << 7) - TT_LOW + 1;
constexpr int TT_NT = 1024, TT_WGS = 256;                     // one workgroup to a compute unit (as two of 512 threads, with twice the tables to make: 57 us instead of 55)

// sum of 2^((v - top) k) of a chunk's values; false: some are not in the table
__device__ __forceinline__ bool tv_table_sum(const TvRaw<bf16_t> *raw, const double *table, TvBits bits, float top, double k, double *out) {
    const unsigned int base = (unsigned int)(uintptr_t)(const __attribute__((address_space(3))) double *)table;
    double sum = 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        double x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned int two = raw[q].w[0][e];
            const tv_ushorts size = __builtin_bit_cast(tv_ushorts, two & 0x7fff7fffu);
            const tv_ushorts of = __builtin_elementwise_min(__builtin_elementwise_sub_sat(size, (tv_ushorts)(TT_LOW - 1)), (tv_ushorts)TT_LAST);
            const unsigned int at = __builtin_bit_cast(unsigned int, (tv_ushorts)(of << 4)) | __builtin_bit_cast(unsigned int, (tv_ushorts)(__builtin_bit_cast(tv_ushorts, two) >> 12)) & 0x00080008u;
            x[2 * e] = *(const __attribute__((address_space(3))) double *)(uintptr_t)(base + (at & 0xffffu));
            x[2 * e + 1] = *(const __attribute__((address_space(3))) double *)(uintptr_t)(base + (at >> 16));
        }
        __builtin_amdgcn_sched_barrier(0);
        sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
    }
    const double all = tv_lane(tv_upto(sum), 63), top_k = top * k;
    // (nothing is left out but what is 2^-200 of the sum, at most)
    if (!(all > 0.0 && top_k > -700.0) || (__any(bits.low >= 0xc3800000u) && !((top + 256.0) * k > 200.0))) return false;
    *out = all * tv_exp2(-top_k);
    return true;
}

// Exponentials of a chunk are taken as 2^(v k - E), E the whole number next to top k: what v k is beyond a whole number has nothing to do with the top, and E goes to the exponent.
// So a value costs 17 instructions, eight of them the polynomial's.
// TABLE (bf16): from the powers of all values in range, where all of the chunk's are.
template <typename T, bool TABLE>
__device__ __forceinline__ TvStat tv_stat(const TvArgs &a, const T *from, int chunk, int lane, float t, const TvRaw<T> *raw, const double *table) {
    const double k = 1.4426950408889634 / (double)t;
    // fp32 bits as signed numbers: the largest is the largest value, if that is not negative, and +inf or more where there is one or a NaN; as unsigned numbers: more than -inf where there is a negative NaN
    const TvBits bits = tv_bits(raw);
    const bool bad = __any(bits.top >= 0x7f800000 || bits.low > 0xff800000u);
    float own = __int_as_float(bits.top);                     // the lane's largest
    if (__any(bits.top < 0)) {                                // (or all of a lane's are negative)
        own = -INFINITY;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[8];
            tv_values(raw[q], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) own = fmaxf(own, v[e]);
        }
    }
    const float top = tv_max_all(own);
    double sum = 0.0;
    int first = INT32_MAX;
    if (t > 0.f && top > -INFINITY && !bad) {
        if constexpr (TABLE) {
            if (t <= FLT_MAX && tv_table_sum(raw, table, bits, top, k, &sum)) return TvStat{top, first, sum};
            sum = 0.0;
        }
        // Against the lane's own largest value: nothing waits for the wavefront's. (One that has none takes the wavefront's, and what it sums up is nothing.)
        const float mine = own > -INFINITY ? own : top, least = tv_least(mine, t);
        const double mk = mine * k, top_k = top * k;
        if (!__any(!((mine - (double)least) * k > 200.0 && fabs(mk) < 4096.0))) {          // what is below the least counts as that: 2^-200 of the sum, at most
            const double e_own = __builtin_rint(mk), e_top = __builtin_rint(top_k), magic = 0x1.8p52 - e_own;
            double c9 = TV_C9;
            asm("" : "+v"(c9));                               // (an instruction takes one constant from scalar registers)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[8];
                tv_values(raw[q], v);
#pragma unroll
                for (int e0 = 0; e0 < 8; e0 += 4) {
                    double d[4], w[4], f[4], y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = (double)tv_at_least(v[e0 + e], least);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = __builtin_fma(d[e], k, magic);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = __builtin_fma(d[e], k, magic - w[e]);
                    tv_poly<4>(f, y, c9);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        tv_pair b = __builtin_bit_cast(tv_pair, y[e]);
                        b[1] += __builtin_bit_cast(tv_pair, w[e])[0] << 20;
                        y[e] = __builtin_bit_cast(double, b);
                    }
                    sum += (y[0] + y[1]) + (y[2] + y[3]);
                }
            }
            // the sum against 2^(top k)
            const double over = e_top - top_k;                // (half a step either way)
            double scale;
            tv_poly<1>(&over, &scale);
            sum = own > -INFINITY ? __builtin_ldexp(sum * scale, (int)(e_own - e_top)) : 0.0;
        } else {                                              // so high a temperature, or such large values, that no fp32 number is that far below the top, or that products are not exact enough
#pragma unroll 1
            for (int q = 0; q < 4; ++q) {
                TvRaw<T> again;
                float y[8];
                tv_load<T, 1>(from, chunk, q, lane, a.vocab, &again);
                tv_values(again, y);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += tv_exp2(((double)y[e] - top) * k);
            }
        }
        sum = tv_lane(tv_upto(sum), 63);
    } else if (t == 0.f) {
#pragma unroll
        for (int q = 3; q >= 0; --q) {
            float v[8];
            tv_values(raw[q], v);
#pragma unroll
            for (int e = 7; e >= 0; --e)
                if (v[e] == top) first = tv_at(chunk, q, lane) + e;
        }
        first = tv_min(first);
    }
    return TvStat{bad ? 0.f : top, first, bad ? (double)NAN : sum};
}

// whether row i of a request has children: if not, its draft's logits are nobody's
__device__ __forceinline__ bool tv_has_children(const TvArgs &a, RowsRange rows, int i, int lane) {
    bool child = false;
    for (int j = i + 1 + lane; j < min(rows.n, KNNSSD_MAX_TREE); j += 64) child = child || a.parents[rows.first + j] == i;
    return __any(child);
}

template <typename T>
__global__ __launch_bounds__(256) void tv_stats_kernel(TvArgs a) {
    const int lane = threadIdx.x & 63;
    int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const bool draft = unit >= a.n_rows * a.chunks;
    if (draft) unit -= a.n_rows * a.chunks;
    const int row = unit / a.chunks, chunk = unit - row * a.chunks;
    if (row >= a.n_rows || (draft && !a.draft)) return;       // (from here on wavefronts are on their own)
    const int r = battn_request(a.row_start, a.n_requests, row);
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int i = row - rows.first;
    if (i < 0 || i >= rows.n || i >= KNNSSD_MAX_TREE) return;
    if (draft && !tv_has_children(a, rows, i, lane)) return;
    const T *from = (const T *)(draft ? a.draft : a.logits) + row * (draft ? a.draft_stride : a.logits_stride);
    TvRaw<T> raw[4];
    tv_load<T, 4>(from, chunk, 0, lane, a.vocab, raw);
    const TvStat stat = tv_stat<T, false>(a, from, chunk, lane, a.temperature[r], raw, nullptr);
    if (lane == 0) a.stats[(size_t)(draft ? a.n_rows : 0) * a.chunks + unit] = stat;
}

// The same of large batches in bf16, with 2^(v k) for all bf16 values of 2^-17 <= |v| < 2^8 in LDS: a value is then seven instructions and a read, its sum against nothing, as such powers
// have room in 64 bits. A workgroup has a run of chunks, a request's behind another's, and makes the table anew where the temperature changes. Of a request's chunks the first
// sixteen of all its rows come first, then the next ones, so that draft's rows that nobody looks at (no children) are no run's alone.
// 284 rows of 152064 tokens in 32 requests: 29.4 us (tv_stats_kernel 34.5), for 19 of which wavefronts live, reading at the rate of memory; of 256 requests of 9 rows, drawn, the whole call 365 us
// for 1.3 GB.
__global__ __launch_bounds__(TT_NT, 4) void tv_stats_table_kernel(TvArgs a) {
    __shared__ double table[2 * TT_LAST + 2];
    __shared__ int inner[KNNSSD_MAX_TREE];                    // 1 + the last request whose row of this number has children
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool drawn = a.draft != nullptr;
    const int sides = drawn ? 2 : 1;
    const long long units = (long long)max(0, min(a.n_rows, a.row_start[a.n_requests])) * sides * a.chunks;
    const int begin = (int)(units * blockIdx.x / gridDim.x), end = (int)(units * (blockIdx.x + 1) / gridDim.x);
    for (int i = tid; i < KNNSSD_MAX_TREE; i += TT_NT) inner[i] = 0;
    float table_t = 0.f;
    for (int at = begin, next; at < end; at = next) {
        const int row0 = at / (sides * a.chunks), r = battn_request(a.row_start, a.n_requests, row0);
        const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
        const int first = rows.first, n = rows.n, per = sides * n;
        const bool inside = row0 >= first && row0 < first + n;
        next = min(end, (inside ? first + n : row0 + 1) * sides * a.chunks);
        if (!inside) continue;
        const int x0 = at - first * sides * a.chunks + wave, x1 = next - first * sides * a.chunks;
        const float t = a.temperature[r];
        auto place = [&](int x, int *j, int *chunk) __attribute__((always_inline)) {
            constexpr int W = TT_NT / 64;
            const int turn = x / (per * W), in = x - turn * per * W, width = min(W, a.chunks - turn * W);
            *j = in / width;
            *chunk = turn * W + in - *j * width;
        };
        // a unit's values on their way; false: nobody looks at them
        auto load = [&](int x, bool known, TvRaw<bf16_t> *raw) __attribute__((always_inline)) {
            if (x >= x1) return false;
            int j, chunk;
            place(x, &j, &chunk);
            const int i = j < n ? j : j - n;
            if (i >= KNNSSD_MAX_TREE || (known && j >= n && __builtin_amdgcn_readfirstlane(inner[i]) != r + 1)) return false;
            tv_load<bf16_t, 4>(j < n ? (const bf16_t *)a.logits + (first + i) * a.logits_stride : (const bf16_t *)a.draft + (first + i) * a.draft_stride, chunk, 0, lane, a.vocab, raw);
            return true;
        };
        TvRaw<bf16_t> raw[4], ahead[4];
        bool here = load(x0, false, raw);
        __syncthreads();
        if (drawn)
            for (int j = 1 + tid; j < min(n, KNNSSD_MAX_TREE); j += TT_NT) {
                const int p = a.parents[first + j];
                if (p >= 0 && p < j) inner[p] = r + 1;
            }
        if (t > 0.f && t <= FLT_MAX && t != table_t) {
            const double k = 1.4426950408889634 / (double)t;
            for (int x = tid; x <= TT_LAST; x += TT_NT) {     // (0: smaller ones and 0; the last: larger ones, -inf)
                const double vk = (double)__uint_as_float((unsigned int)(x + TT_LOW - 1) << 16) * k, y = tv_exp2(fmin(vk, 1000.0));
                const bool beyond = x == TT_LAST || vk > 1000.0;
                table[2 * x] = x == 0 || beyond ? (double)NAN : y;
                table[2 * x + 1] = x == 0 ? (double)NAN : beyond ? 0.0 : 1.0 / y;
            }
            table_t = t;
        }
        __syncthreads();
        for (int x = x0; x < x1; x += TT_NT / 64) {
            const bool then = load(x + TT_NT / 64, true, ahead);
            int j, chunk;
            place(x, &j, &chunk);
            const int i = j < n ? j : j - n;
            if (here && (j < n || __builtin_amdgcn_readfirstlane(inner[i]) == r + 1)) {
                const bf16_t *from = j < n ? (const bf16_t *)a.logits + (first + i) * a.logits_stride : (const bf16_t *)a.draft + (first + i) * a.draft_stride;
                const TvStat stat = tv_stat<bf16_t, true>(a, from, chunk, lane, t, raw, table);
                if (lane == 0) a.stats[((size_t)(j < n ? 0 : a.n_rows) + first + i) * a.chunks + chunk] = stat;
            }
            here = then;
#pragma unroll
            for (int q = 0; q < 4; ++q) raw[q] = ahead[q];
        }
    }
}

// a row's chunks put together by a group of `width` lanes, four chunks a lane at a time
__device__ __forceinline__ TvRow tv_join(const TvStat *s, int chunks, double k, int in, int width) {
    constexpr int U = 4;
    TvRow row{-INFINITY, INT32_MAX, 0.0};
    for (int c0 = in; c0 - in < chunks; c0 += U * width) {    // (the same number of times for all of the group)
        float top[U], most = row.top;
        int first[U];
        double sum[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int c = c0 + j * width;
            top[j] = -INFINITY;
            first[j] = INT32_MAX;
            sum[j] = 0.0;
            if (c < chunks) {
                const TvStat one = s[c];
                top[j] = one.top;
                first[j] = one.first;
                sum[j] = one.sum;
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j) most = fmaxf(most, top[j]);
        most = tv_max(most, width);
        if (most > row.top) {
            if (row.top > -INFINITY) row.sum *= tv_exp2(((double)row.top - most) * k);
            row.top = most;
            row.first = INT32_MAX;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (j > 0 && c0 - in + j * width >= chunks) break;
            if (top[j] > -INFINITY) row.sum += sum[j] * tv_exp2(((double)top[j] - row.top) * k);
            else if (sum[j] != sum[j]) row.sum = sum[j];
            if (top[j] == row.top) row.first = min(row.first, first[j]);
        }
    }
    row.sum = tv_sum(row.sum, width);
    row.first = tv_min(row.first, width);
    if (row.sum != row.sum || row.top == -INFINITY) row.top = NAN;
    return row;
}

// weights of N values (and of the draft's, w)
template <int N, bool DRAFT>
__device__ __forceinline__ void tv_weigh(const TvWeigh &s, const float *v, const float *w, double *out) {
    double d[N], y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] = (double)tv_at_least(v[e], s.p_least) - (double)s.p_top;
    tv_exp2_near<N>(d, s.k, y);
#pragma unroll
    for (int e = 0; e < N; ++e) out[e] = v[e] >= s.p_least ? s.p_each * y[e] : 0.0;
    if constexpr (DRAFT) {
#pragma unroll
        for (int e = 0; e < N; ++e) d[e] = (double)tv_at_least(w[e], s.q_least) - (double)s.q_top;
        tv_exp2_near<N>(d, s.k, y);
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = __builtin_fmax(w[e] >= s.q_least ? __builtin_fma(-s.q_each, y[e], out[e]) : out[e], 0.0);
    }
}

// sum of the weights of eight tokens (and the draft's)
template <typename T, bool DRAFT>
__device__ __forceinline__ double tv_weights8(const TvWeigh &s, const TvRaw<T> &p, const TvRaw<T> &q) {
    float v[8], w[8];
    tv_values(p, v);
    if constexpr (DRAFT) tv_values(q, w);
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
        double y[4];
        tv_weigh<4, DRAFT>(s, v + e, w + e, y);
        sum += (y[0] + y[1]) + (y[2] + y[3]);
    }
    return sum;
}

// of eight tokens from `at` on, those that were rejected are ruled out
__device__ __forceinline__ void tv_without(const int *rejected, int n, int at, TvRaw<float> &raw) {
    for (int x = 0; x < n; ++x) {
        const int d = rejected[x] - at;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d == e) raw.w[e >> 2][e & 3] = 0xff800000u;
    }
}
__device__ __forceinline__ void tv_without(const int *rejected, int n, int at, TvRaw<bf16_t> &raw) {
    for (int x = 0; x < n; ++x) {
        const int d = rejected[x] - at;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (d == e) raw.w[0][e >> 1] = (raw.w[0][e >> 1] & (e & 1 ? 0xffffu : 0xffff0000u)) | (e & 1 ? 0xff800000u : 0xff80u);
    }
}

// Rounds: a rejected draw needs the sum over its whole row before the walk can go on. The walk of `round` stops there if a launch of tv_sum_kernel and another round follow
// (`more`), and goes on in that; one that has no further round takes the sums that it still needs by itself. The first wavefront walks: steps are short, and a compute unit's
// other wavefronts would only be in its way.
template <typename T>
__global__ __launch_bounds__(TV_NT) void tv_walk_kernel(TvArgs a, int round, int more) {
    __shared__ int parent[KNNSSD_MAX_TREE], token[KNNSSD_MAX_TREE], u_bits[KNNSSD_MAX_TREE];
    __shared__ TvRow p_row[KNNSSD_MAX_TREE], q_row[KNNSSD_MAX_TREE];
    __shared__ double p_at[KNNSSD_MAX_TREE], q_at[KNNSSD_MAX_TREE], chunk_sum[TV_MAX_CHUNKS], part[2][TV_WAVES];
    __shared__ bool inner[KNNSSD_MAX_TREE];                   // has children
    __shared__ struct { double c, target; int node, n_rejected, chunk; bool summed, ended; } now;
    __shared__ int found[TV_WAVES], held[TV_WAVES];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int n = min(rows.n, KNNSSD_MAX_TREE);
    const float t = a.temperature[r];
    const bool drawn = a.draft != nullptr, greedy = t == 0.f;
    int node = 0, last = 0, kept = 1;                         // where the walk is, its child that was tried last, rows taken
    double c = 0.0;
    if (round > 0) {
        if (!a.states[r].waits) return;
        node = a.states[r].node; last = a.states[r].last; kept = a.states[r].kept; c = a.states[r].c;
    } else if (n == 0 || !(t >= 0.f && t <= FLT_MAX)) {
        for (int i = tid; i < rows.n; i += TV_NT) a.path[rows.first + i] = -1;
        if (tid == 0) {
            a.n_path[r] = 0;
            a.next[r] = -1;
            if (more) a.states[r].waits = 0;
        }
        return;
    }
    const double k = greedy ? 0.0 : 1.4426950408889634 / (double)t;
    const T *logits = (const T *)a.logits + rows.first * a.logits_stride, *draft = (const T *)a.draft + (drawn ? rows.first * a.draft_stride : 0);
    const TvStat *p_stats = a.stats + (size_t)rows.first * a.chunks, *q_stats = p_stats + (size_t)a.n_rows * a.chunks;
    if (round > 0) {
        for (int i = tid; i < n; i += TV_NT) {
            const TvNode o = a.nodes[rows.first + i];
            parent[i] = o.parent; token[i] = o.token; u_bits[i] = o.u; inner[i] = o.inner;
            p_row[i] = o.p; q_row[i] = o.q; p_at[i] = o.p_at; q_at[i] = o.q_at;
        }
        for (int x = tid; x < a.chunks; x += TV_NT) chunk_sum[x] = a.sums[(size_t)r * a.chunks + x];
        __syncthreads();
    } else {
        int p[TV_EACH], x[TV_EACH];
        float pv[TV_EACH], qv[TV_EACH];
#pragma unroll
        for (int e = 0; e < TV_EACH; ++e) {
            const int i = tid + e * TV_NT;
            p[e] = -1;
            if (i >= n) continue;
            p[e] = a.parents[rows.first + i];
            x[e] = a.tokens[rows.first + i];
            u_bits[i] = __float_as_int(a.u_accept[rows.first + i]);
            if (!(p[e] >= 0 && p[e] < i && (unsigned)x[e] < (unsigned)a.vocab)) p[e] = -1;          // (a token that is none never passes)
            parent[i] = p[e];
            token[i] = x[e];
            inner[i] = false;
            if (p[e] < 0) continue;                           // (on their way while the rows are put together)
            pv[e] = load_as_float(logits + p[e] * a.logits_stride, x[e]);
            if (drawn) qv[e] = load_as_float(draft + p[e] * a.draft_stride, x[e]);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < TV_EACH; ++e)
            if (p[e] >= 0) inner[p[e]] = true;
        for (int i = tid; i < rows.n; i += TV_NT) a.path[rows.first + i] = i == 0 ? 0 : -1;
        __syncthreads();
        // the rows' sums put together, a group of lanes each; the draft's where it has been asked for any
        const int jobs = drawn ? 2 * n : n;
        int width = 64;
        while (width > 4 && (width * jobs > TV_NT || width >= 2 * a.chunks)) width >>= 1;
        const int in = tid & (width - 1);
        for (int j = tid / width; j < jobs; j += TV_NT / width) {
            const bool of_draft = j >= n;
            const int i = of_draft ? j - n : j;
            if (of_draft && !inner[i]) continue;
            const TvRow row = tv_join((of_draft ? q_stats : p_stats) + (size_t)i * a.chunks, a.chunks, k, in, width);
            if (in == 0) (of_draft ? q_row : p_row)[i] = row;
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < TV_EACH; ++e) {
            const int i = tid + e * TV_NT;
            if (p[e] < 0) continue;
            auto share = [&](const TvRow &row, float v) __attribute__((always_inline)) { return greedy ? (x[e] == row.first ? 1.0 : 0.0) : tv_exp2(((double)v - row.top) * k) / row.sum; };
            p_at[i] = share(p_row[p[e]], pv[e]);
            if (drawn) q_at[i] = share(q_row[p[e]], qv[e]);
        }
        __syncthreads();
    }

    bool summed = round > 0;                                  // chunk_sum has the node's weights
    while (true) {
        if (wave == 0) {
            double left = 1.0;                                // what of p is left
            bool waits = false, lost = false;                 // for the sum over a row; at a row without a distribution
            bool first = c == 0.0;                            // nothing has been rejected at the node (what is left may still be 1 behind a token of less than 2^-53)
            if (summed) {
                left = 0.0;
                for (int x = lane; x < a.chunks; x += 64) left += chunk_sum[x];
                left = tv_sum(left);
            }
            // a lane has a row of the 64 that the walk is among: whether it is taken if it is the first that is tried, whether it has children, a distribution
            int seg = -1, par = -1, tok = 0;
            float u_of = 0.f;
            double p_of = 0.0, q_of = 1.0;
            unsigned long long taken = 0, with_children = 0, without_one = 0;
            auto among = [&](int s) __attribute__((always_inline)) {
                seg = s;
                const int i = min(s * 64 + lane, n - 1);
                par = s * 64 + lane < n ? parent[i] : -1;
                tok = token[i];
                u_of = __int_as_float(u_bits[i]);
                p_of = p_at[i];
                if (drawn) q_of = q_at[i];
                const bool children = inner[i];
                taken = __ballot(p_of > u_of * q_of);
                with_children = __ballot(children);
                without_one = __ballot(p_row[i].top != p_row[i].top || (drawn && children && q_row[i].top != q_row[i].top));
            };
            among(node >> 6);
            bool goes_on = with_children >> (node & 63) & 1;
            lost = without_one >> (node & 63) & 1;
            if (last >> 6 > seg) among(last >> 6);
            while (!waits && !lost && goes_on) {
                const unsigned long long match = __ballot(par == node && seg * 64 + lane > last);
                if (!match) {
                    if ((seg + 1) * 64 >= n) break;
                    among(seg + 1);
                    continue;
                }
                const int l = __builtin_ctzll(match), child = seg * 64 + l;
                last = child;
                bool take = taken >> l & 1;
                double px = 0.0, qx = 1.0;
                if (!first || !take) {
                    const double u = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(u_of), l));
                    px = tv_lane(p_of, l);
                    qx = tv_lane(q_of, l);
                    if (!drawn && !first) {                   // the same token again: it has been rejected
                        const int x = __builtin_amdgcn_readlane(tok, l);
                        if (__any(par == node && tok == x && lane < l)) px = 0.0;
                        for (int i = (node & ~63) + lane; i < seg * 64; i += 64)
                            if (__any(parent[i] == node && token[i] == x)) px = 0.0;
                    }
                    take = px > (c + u * left) * qx;
                }
                if (take) {
                    node = child;
                    if (lane == 0) a.path[rows.first + kept] = child;
                    ++kept;
                    c = 0.0;
                    left = 1.0;
                    first = true;
                    summed = false;
                    goes_on = with_children >> l & 1;
                    lost = without_one >> l & 1;
                } else if (!drawn) {
                    left -= px;
                    first = false;
                } else if (qx > 0.0) {                        // (a token that the draft cannot have drawn says nothing about its distribution)
                    c += left;
                    first = false;
                    waits = !greedy;
                    left = 1.0;                               // (greedy: p and q are each all on one token, not the same: p stays)
                }
            }
            if (lane == 0) {
                now.node = node;
                now.c = c;
                now.summed = summed;
                now.ended = !waits;
                now.n_rejected = 0;
                if (!waits) {
                    a.n_path[r] = kept;
                    if (more) a.states[r].waits = 0;
                    if (lost || greedy) a.next[r] = lost ? -1 : p_row[node].first;
                    if (lost || greedy) now.node = -1;
                } else if (more) {
                    a.states[r] = TvState{TvWeigh{p_row[node].top, q_row[node].top, tv_least(p_row[node].top, t), tv_least(q_row[node].top, t), 1.0 / p_row[node].sum,
                                                  c / q_row[node].sum, k}, c, node, last, kept, 1};
                    a.n_path[r] = kept;
                }
            }
        }
        __syncthreads();
        if (now.ended) break;
        node = now.node;
        c = now.c;
        if (more) {
            if (round == 0)
                for (int i = tid; i < n; i += TV_NT) {
                    TvNode &o = a.nodes[rows.first + i];
                    o.p = p_row[i]; o.q = q_row[i]; o.p_at = p_at[i]; o.q_at = q_at[i];
                    o.parent = parent[i]; o.token = token[i]; o.u = u_bits[i]; o.inner = inner[i];
                }
            return;
        }
        const TvWeigh w{p_row[node].top, q_row[node].top, tv_least(p_row[node].top, t), tv_least(q_row[node].top, t), 1.0 / p_row[node].sum, c / q_row[node].sum, k};
        // four wavefronts to a chunk, the next one's values on their way
        const T *p = logits + node * a.logits_stride, *q = draft + node * a.draft_stride;
        TvRaw<T> p_raw, q_raw, p_next, q_next;
        auto load = [&](int x, TvRaw<T> &to_p, TvRaw<T> &to_q) __attribute__((always_inline)) {
            if (x >= a.chunks) return;
            tv_load<T, 1>(p, x, wave & 3, lane, a.vocab, &to_p);
            tv_load<T, 1>(q, x, wave & 3, lane, a.vocab, &to_q);
        };
        load(wave / 4, p_raw, q_raw);
        for (int x0 = 0, b = 0; x0 < a.chunks; x0 += TV_WAVES / 4, b ^= 1) {
            const int x = x0 + wave / 4;
            load(x + TV_WAVES / 4, p_next, q_next);
            double sum = 0.0;
            if (x < a.chunks) sum = tv_lane(tv_upto(tv_weights8<T, true>(w, p_raw, q_raw)), 63);
            p_raw = p_next;
            q_raw = q_next;
            if (lane == 0) part[b][wave] = sum;
            __syncthreads();
            if (x < a.chunks && (tid & 255) == 0) chunk_sum[x] = (part[b][wave] + part[b][wave + 1]) + (part[b][wave + 2] + part[b][wave + 3]);
        }
        __syncthreads();
        summed = true;
    }
    node = now.node;
    if (node < 0) return;

    // the next token: of max(p - c q, 0), or of p without the rejected tokens
    c = now.c;
    summed = now.summed;
    int *rejected = u_bits, gone = 0;
    const T *p = logits + node * a.logits_stride, *q = draft + node * a.draft_stride;
    const TvWeigh w{p_row[node].top, summed ? q_row[node].top : 0.f, tv_least(p_row[node].top, t), summed ? tv_least(q_row[node].top, t) : 0.f,
                    summed ? 1.0 / p_row[node].sum : 1.0, summed ? c / q_row[node].sum : 0.0, k};
    if (!summed) {
        const TvStat *own = p_stats + (size_t)node * a.chunks;
        // (a chunk all of whose tokens are below the least has no weight, as it has none where a token is picked: under a target of 0 it would be the first one)
        for (int x = tid; x < a.chunks; x += TV_NT) chunk_sum[x] = own[x].top >= w.p_least ? own[x].sum * tv_exp2(((double)own[x].top - w.p_top) * k) : 0.0;
        if (!drawn && inner[node])
            for (int i = tid; i < n; i += TV_NT)
                if (parent[i] == node) rejected[atomicAdd(&now.n_rejected, 1)] = token[i];       // (in any order: all of them get a weight of 0)
        __syncthreads();
        gone = now.n_rejected;
        for (int i0 = 0, b = 0; i0 < gone; i0 += TV_WAVES / 4, b ^= 1) {      // chunks with rejected tokens anew (some more than once, to the same end)
            const int i = i0 + wave / 4, x = i < gone ? rejected[i] / TV_CHUNK : 0;
            double sum = 0.0;
            if (i < gone) {
                TvRaw<T> raw;
                tv_load<T, 1>(p, x, wave & 3, lane, a.vocab, &raw);
                tv_without(rejected, gone, tv_at(x, wave & 3, lane), raw);
                sum = tv_lane(tv_upto(tv_weights8<T, false>(w, raw, raw)), 63);
            }
            if (lane == 0) part[b][wave] = sum;
            __syncthreads();
            if (i < gone && (tid & 255) == 0) chunk_sum[x] = (part[b][wave] + part[b][wave + 1]) + (part[b][wave + 2] + part[b][wave + 3]);
        }
        if (gone) __syncthreads();
    }
    // the chunk that the target lies in, or the last one with a weight: a lane of the first wavefront has some neighbouring ones
    if (wave == 0) {
        constexpr int EACH = TV_MAX_CHUNKS / 64;
        double mine = 0.0, each[EACH];
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            const int x = lane * EACH + j;
            each[j] = x < a.chunks ? chunk_sum[x] : 0.0;
            mine += each[j];
        }
        const double upto = tv_upto(mine), target = (double)a.u_next[r] * tv_lane(upto, 63);
        double run = upto - mine, before = 0.0, held_before = 0.0;
        int chunk = -1, held_chunk = -1;
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
            if (each[j] > 0.0) {
                held_chunk = lane * EACH + j;
                held_before = run;
                if (chunk < 0 && run + each[j] > target) {
                    chunk = held_chunk;
                    before = run;
                }
            }
            run += each[j];
        }
        const unsigned long long past = __ballot(chunk >= 0), any = __ballot(held_chunk >= 0);
        if (past || any) {
            if (lane == (past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any))) {
                now.chunk = past ? chunk : held_chunk;
                now.target = target - (past ? before : held_before);
            }
        } else if (lane == 0) {
            now.chunk = -1;
            a.next[r] = -1;
        }
    }
    __syncthreads();
    const int chunk = now.chunk;
    if (chunk < 0) return;
    // the chunk's first token that the weights up to and with it are more than the target, or (roundings) its last one with a weight: a thread has neighbouring tokens
    const double target = now.target;
    const int at = chunk * TV_CHUNK + TV_PICK * tid;
    double x[TV_PICK], sum = 0.0;
    float pv[TV_PICK], qv[TV_PICK];
#pragma unroll
    for (int e = 0; e < TV_PICK; ++e) {
        pv[e] = at + e < a.vocab ? load_as_float(p, at + e) : -INFINITY;
        qv[e] = summed && at + e < a.vocab ? load_as_float(q, at + e) : -INFINITY;
    }
    for (int i = 0; i < gone; ++i) {
        const int d = rejected[i] - at;
#pragma unroll
        for (int e = 0; e < TV_PICK; ++e) pv[e] = d == e ? -INFINITY : pv[e];
    }
    tv_weigh<TV_PICK, true>(w, pv, qv, x);                    // (nothing of q where it is -inf)
#pragma unroll
    for (int e = 0; e < TV_PICK; ++e) sum += x[e];
    const double upto = tv_upto(sum);
    if (lane == 63) part[0][wave] = upto;
    __syncthreads();
    double run = 0.0;
    for (int i = 0; i < wave; ++i) run += part[0][i];
    run += upto - sum;
    int mine = INT32_MAX, with = -1;
#pragma unroll
    for (int e = 0; e < TV_PICK; ++e) {
        run += x[e];
        if (x[e] > 0.0) {
            with = at + e;
            if (mine == INT32_MAX && run > target) mine = at + e;
        }
    }
    const unsigned long long past = __ballot(mine != INT32_MAX), any = __ballot(with >= 0);       // (tokens are in the order of the lanes)
    mine = past ? __builtin_amdgcn_readlane(mine, __builtin_ctzll(past)) : INT32_MAX;
    with = any ? __builtin_amdgcn_readlane(with, 63 - __builtin_clzll(any)) : -1;
    if (lane == 0) {
        found[wave] = mine;
        held[wave] = with;
    }
    __syncthreads();
    if (tid == 0) {
        for (int i = 0; i < TV_WAVES; ++i) {
            mine = min(mine, found[i]);
            with = max(with, held[i]);
        }
        a.next[r] = mine != INT32_MAX ? mine : with;
    }
}

// Sums of max(p - c q, 0) over the chunks of the rows at which walks wait, a workgroup each.
template <typename T>
__global__ __launch_bounds__(256) void tv_sum_kernel(TvArgs a) {
    __shared__ double part[4];
    const int chunk = blockIdx.x, r = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const TvState s = a.states[r];
    if (!s.waits) return;
    const long long row = rows_of(a.row_start, r, a.n_rows).first + s.node;
    TvRaw<T> p, q;
    tv_load<T, 1>((const T *)a.logits + row * a.logits_stride, chunk, wave, lane, a.vocab, &p);
    tv_load<T, 1>((const T *)a.draft + row * a.draft_stride, chunk, wave, lane, a.vocab, &q);
    const double sum = tv_lane(tv_upto(tv_weights8<T, true>(s.w, p, q)), 63);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(size_t)r * a.chunks + chunk] = (part[0] + part[1]) + (part[2] + part[3]);
}

}  // namespace ks
