// What the attention kernels of a batch share: arguments, operands, loads to LDS, and partial results of a group of (row, head) pairs.
#pragma once
#include <type_traits>

#include "kernels_pages.h"
#include "rows_range.h"

namespace ks {

// ints that nothing writes while the kernel runs, by scalar loads where the index is the same for all lanes
typedef const __attribute__((address_space(4))) int *const_ints;

struct BattnArgs {
    const void *q, *k, *v;
    void *out;
    long long q_stride, out_stride;             // rows of q and out
    long long k_stride, v_stride;               // rows of k and v (prompts)
    long long page_stride, head_stride, pos_stride;
    const_ints table, row_start, kv_len;        // (kv_len, table: pages)
    int n_requests, n_rows, width, shift, n_pages;
    int H, Hkv, group;
    float scale2;                               // scale * log2(e): softmax in powers of two
    void *ws;
};

// request of row t < row_start[n], by bisection
__device__ __forceinline__ int battn_request(const_ints row_start, int n, int t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// positions of request r: what its table can hold at most, and no more than 2^30
__device__ __forceinline__ int battn_len(const BattnArgs &a, int r) {
    return (int)min((long long)min(max(a.kv_len[r], 0), 1 << 30), (long long)a.width << a.shift);
}

// element where position p of request r begins for kv head h. A page id outside the cache reads page 0 instead.
__device__ __forceinline__ long long battn_paged(const BattnArgs &a, int r, int h, int p) {
    const int g = a.table[(size_t)r * a.width + (p >> a.shift)];
    return ((unsigned)g < (unsigned)a.n_pages ? g : 0) * a.page_stride + h * a.head_stride + (p & ((1 << a.shift) - 1)) * a.pos_stride;
}

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
#define BATTN_LDS(p) ((__attribute__((address_space(3))) char *)(p))

// lane i's value, known to be the same everywhere (scalar registers, scalar loads)
__device__ __forceinline__ long long battn_lane(long long v, int i) {
    return (long long)(unsigned int)__builtin_amdgcn_readlane((int)v, i) | (long long)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32;
}

// the same for a value that the compiler has worked out in vector registers (64-bit comparisons and choices, conversions) though it is the same for all
__device__ __forceinline__ int battn_same(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ long long battn_same(long long v) { return battn_lane(v, 0); }

// 64 lanes' 16 bytes from base + off (bytes) to LDS, lane by lane behind lds_off. Not counted by the compiler: battn_wait. (s_nop: a
// base that the vector unit has just written may be read five states later.)
__device__ __forceinline__ void battn_dma(const void *base, unsigned int off, unsigned int lds_off) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(battn_same((long long)(uintptr_t)base)), "s"(battn_same((int)lds_off)) : "memory");
}
template <int KEEP> __device__ __forceinline__ void battn_wait() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(KEEP) : "memory"); }
// a workgroup's meeting that leaves loads in flight (this wavefront's LDS reads have returned)
__device__ __forceinline__ void battn_meet() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}
// a * b rounded, also where the compiler could fold the product into a following sum
__device__ __forceinline__ float battn_rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

constexpr int BF_WGS = 512;                                   // most runs that a batch is dealt out in: two workgroups per compute unit
constexpr int BF_PAD = 4;                                     // floats behind a pair's HD values: its exponent, its sum
typedef float f32x4_t __attribute__((ext_vector_type(4)));

template <int HD> __host__ __device__ constexpr size_t battn_few_slot(int pairs) { return (size_t)pairs * (HD + BF_PAD); }      // floats of a partial result
// a group that begins in a run and does not end there: the runs that hold it, its first row's request, kv head, first pair and pairs
struct FewMerge { int runs, r0, kvh, pair, pairs; };
__host__ __device__ constexpr size_t battn_few_merges() { return BF_WGS * 32; }
static_assert(sizeof(FewMerge) <= 32, "");

// Eight fp32 values as NP bf16 operands: rounded to nearest (1), or cut three times into exact parts (3). Weights of bf16 queries are rounded: by half a step, 2^-8, each, so an
// output by at most 2^-8 of sum(weight |value|), as its own rounding to bf16 does (errors against 64 bits of 0.0020 to 0.0023 of the outputs' size, with fp32 weights 0.0016 to 0.0017).
// Exact weights would take three products for one in the second half of what bounds the tiles.
template <int NP>
__device__ __forceinline__ void battn_planes(const float *v, bf16x8_t *out) {
    if constexpr (NP == 1) {
        out[0] = __builtin_bit_cast(bf16x8_t, u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
    } else {
        float rest[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) rest[e] = v[e];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            u32x4_t w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * e + 1]), __float_as_uint(rest[2 * e]), 0x07060302u);
                rest[2 * e] -= __uint_as_float(w[e] << 16);
                rest[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
            }
            out[p] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
}

// x / d for 0 <= x < 2^53 and d > 0, the same for all lanes: many times shorter than a division of 64-bit integers
__device__ __forceinline__ long long battn_divide(long long x, long long d) {
    long long q = (long long)((double)x / (double)d);
    if (q * d > x) --q;
    if ((q + 1) * d <= x) ++q;
    return battn_same(q);
}

// run that has a unit, where the first rem runs have q + 1 units and the others q
__device__ __forceinline__ int battn_run_of(long long unit, long long q, long long rem) {
    const long long longer = rem * (q + 1);
    return (int)(unit < longer ? battn_divide(unit, q + 1) : rem + battn_divide(unit - longer, q));
}

// A workgroup's run. Workgroups are dealt round the eight XCDs; runs next to each other, which share keys and values or a group whose partial results are
// joined, go to one of them (the grids are multiples of eight).
__device__ __forceinline__ int battn_run() { return (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)); }

// V values of one pair, divided by the sum of its weights
template <int V, int HD, int NP>
__device__ __forceinline__ void battn_few_out(const BattnArgs &a, int r0, int kvh, int pair, int d, float *v, float sum) {
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] *= inv;
    const long long at = (long long)(r0 + pair / a.group) * a.out_stride + (kvh * a.group + pair % a.group) * HD + d;
    if constexpr (NP == 1) store_values<V>((bf16_t *)a.out + at, v);
    else store_values<V>((float *)a.out + at, v);
}

// Joins the partial results of a group. HD/4 lanes have a pair, four values each, and take its runs' results one after the other, four requested at a
// time; where the group lies in more than eight runs, four such teams share them. In a launch of its own: the last workgroup of a group doing it inside
// the first launch had to fetch up to 32 runs' results of all pairs by itself, one memory latency after the other (two requests at
// 100 000 positions: 286 us in all, 168 us in two launches).
constexpr int BM_NT = 256;
template <int HD> __host__ __device__ constexpr int battn_merge_teams() { return BM_NT * 4 / HD; }
template <int HD, int NP>
__global__ __launch_bounds__(BM_NT) void battn_merge_kernel(BattnArgs a, int slot_pairs) {
    constexpr int LP = HD / 4, TEAMS = battn_merge_teams<HD>(), MROW = HD + BF_PAD, U = 4;
    __shared__ f32x4_t part[TEAMS][LP];
    __shared__ float part_top[TEAMS], part_sum[TEAMS];
    const int run = battn_run();
    const FewMerge m = ((const FewMerge *)a.ws)[run];
    if (m.runs == 0) return;                                  // the whole workgroup
    const int lane = threadIdx.x % LP, team = threadIdx.x / LP;
    const int subs = m.runs > 8 ? 4 : 1, sub = team & (subs - 1), at_once = TEAMS / subs;
    const size_t slot = battn_few_slot<HD>(slot_pairs);
    for (int p0 = blockIdx.y * at_once; p0 < m.pairs; p0 += gridDim.y * at_once) {
        const int p = p0 + team / subs;
        // run x's partial result is its second one (a group that begins there) for the first run, its first one for the others
        const float *first = (const float *)((const char *)a.ws + battn_few_merges()) + 2 * run * slot + min(p, m.pairs - 1) * MROW;
        float top = -INFINITY, sum = 0.f;
        f32x4_t v{0.f, 0.f, 0.f, 0.f};
        for (int x = sub; x < m.runs; x += subs * U) {
            float at[U], l[U];
            f32x4_t w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int y = x + subs * u;
                at[u] = -INFINITY;
                l[u] = 0.f;
                if (y < m.runs) {
                    const float *from = first + (2 * y + (y == 0)) * slot;
                    at[u] = from[HD];
                    l[u] = from[HD + 1];
                    w[u] = *reinterpret_cast<const f32x4_t *>(from + lane * 4);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (l[u] == 0.f) continue;                    // nothing seen (what was seen has a weight of 1 at least, or is NaN)
                const float now = fmaxf(top, at[u]), k0 = __builtin_amdgcn_exp2f(top - now), k1 = __builtin_amdgcn_exp2f(at[u] - now);
                top = now;
                sum = sum * k0 + l[u] * k1;
                v = v * k0 + w[u] * k1;
            }
        }
        if (subs > 1) {
            part[team][lane] = v;
            if (lane == 0) { part_top[team] = top; part_sum[team] = sum; }
            __syncthreads();
            if (sub == 0) {
                for (int x = 1; x < subs; ++x) top = fmaxf(top, part_top[team + x]);
                sum = 0.f;
                v = f32x4_t{0.f, 0.f, 0.f, 0.f};
                for (int x = 0; x < subs; ++x) {
                    const float k = part_top[team + x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(part_top[team + x] - top);
                    sum = fmaf(part_sum[team + x], k, sum);
                    v += part[team + x][lane] * k;
                }
            }
            __syncthreads();
        }
        if (sub == 0 && p < m.pairs) {
            float out[4] = {v[0], v[1], v[2], v[3]};
            battn_few_out<4, HD, NP>(a, m.r0, m.kvh, m.pair + p, lane * 4, out, sum);
        }
    }
}

}  // namespace ks
