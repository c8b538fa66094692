// Attention of a batch's rows over pages (PAGED) or over their own prompts' rows.
#pragma once
#include <type_traits>

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
    int few_rows;                               // requests of up to so many rows are battn_few_kernel's
    void *ws;
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

// positions of request r: what its table can hold at most, and no more than 2^30
__device__ __forceinline__ int battn_len(const BattnArgs &a, int r) {
    return (int)min((long long)min(max(a.kv_len[r], 0), 1 << 30), (long long)a.width << a.shift);
}

// element where position p of request r begins for kv head h. A page id outside the cache reads page 0 instead.
__device__ __forceinline__ long long battn_paged(const BattnArgs &a, int r, int h, int p) {
    const int g = a.table[(size_t)r * a.width + (p >> a.shift)];
    return ((unsigned)g < (unsigned)a.n_pages ? g : 0) * a.page_stride + h * a.head_stride + (p & ((1 << a.shift) - 1)) * a.pos_stride;
}

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

// ------------------------------------------------------------------------------------------
// Many rows, bf16: tiles of 128 (row, head) pairs of one kv head, 32 per wavefront, on the matrix cores.
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane keeps one pair from the scores to the output: the
// accumulators of S^T (position 8(i/4) + 4(lane/32) + i%4 of pair lane%32 in register i) are, rounded and packed as they lie, the operand of the
// second product, whose other operand takes the values' positions in the same order by transposing reads of LDS. Nothing is
// exchanged between lanes but one maximum per block.
// Keys and values come in blocks of 64 positions straight to LDS, one block ahead; 16-byte pieces of a row are stored in an order
// (exclusive or with the row's number) in which neither the keys' reads (32 rows, two pieces each) nor the values' (4 rows, 32
// bytes each) meet in a bank.
// ------------------------------------------------------------------------------------------
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
#define BATTN_LDS(p) ((__attribute__((address_space(3))) char *)(p))
typedef const __attribute__((address_space(4))) int *const_ints;        // read by scalar loads

constexpr int BT_PAIRS = 128, BT_CH = 64;

// 64 lanes' 16 bytes from base + off (bytes) to LDS, lane by lane behind lds_off. Not counted by the compiler: battn_wait. (s_nop: a
// base that the vector unit has just written may be read five states later.)
__device__ __forceinline__ void battn_dma(const void *base, unsigned int off, unsigned int lds_off) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(lds_off) : "memory");
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

// Tile `index` of the batch: its request and its number in there; false behind the last. Every wavefront for itself, 64 requests at a time.
__device__ __forceinline__ bool battn_find_tile(const BattnArgs &a, int index, int &r_out, int &tile_out, int &tiles_out) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int r0 = 0; r0 < a.n_requests; r0 += 64) {
        const int r = r0 + lane;
        int mine = 0;
        if (r < a.n_requests) {
            const long long n = min(a.row_start[r + 1], a.n_rows) - max(a.row_start[r], 0);
            if (n > a.few_rows) mine = (int)((n * a.group + BT_PAIRS - 1) / BT_PAIRS);
        }
        int upto = mine;
        for (int off = 1; off < 64; off <<= 1) {
            const int u = __shfl_up(upto, off);
            if (lane >= off) upto += u;
        }
        const unsigned long long past = __ballot(index < before + upto);
        if (past) {
            const int src = __builtin_ctzll(past);
            r_out = r0 + src;
            tiles_out = __builtin_amdgcn_readlane(mine, src);
            tile_out = index - before - (__builtin_amdgcn_readlane(upto, src) - tiles_out);
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

template <int HD> constexpr int battn_tile_lds() { return 2 * 2 * BT_CH * HD * 2; }

template <int HD, bool PAGED>
__global__ __launch_bounds__(256, 2) void battn_tile_kernel(BattnArgs a) {
    constexpr int KS = HD / 16, DT = HD / 32, SL = HD / 8, RB = HD * 2;
    constexpr int KV = BT_CH * RB;                            // bytes of a block's keys (or values)
    constexpr int ROWS = 64 / SL, NI = KV / 1024 / 4;         // rows a wavefront's load covers, loads per wavefront for the keys
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int kvh = blockIdx.x % a.Hkv;                       // (a kv head's tiles run behind few L2s)
    int r, tile, n_tiles;
    if (!battn_find_tile(a, blockIdx.x / a.Hkv, r, tile, n_tiles)) return;
    tile = n_tiles - 1 - tile;                                // long ones first
    const int r0 = max(a.row_start[r], 0), n = min(a.row_start[r + 1], a.n_rows) - r0;
    const int len = PAGED ? battn_len(a, r) : n;
    const int base = len - n;                                 // position of the request's first new row
    const long long pairs = (long long)n * a.group, p0 = (long long)tile * BT_PAIRS;
    const int wave_first = (int)((p0 + wave * 32) / a.group);                                                  // the wavefront's first row
    const int wave_last = (int)(min(p0 + wave * 32 + 31, pairs - 1) / a.group);                                  // ... and last one
    const int tile_last = (int)(min(p0 + BT_PAIRS - 1, pairs - 1) / a.group);
    const int n_blocks = base + tile_last < 0 ? 0 : (base + tile_last) / BT_CH + 1;
    const long long pair = p0 + wave * 32 + col;
    const bool live = pair < pairs;
    const int row = (int)(min(pair, pairs - 1) / a.group), g = (int)(min(pair, pairs - 1) % a.group);
    const int limit = base + row;                             // the lane's last visible position
    const int last = len - 1;
    const unsigned int l0 = (unsigned int)(uintptr_t)BATTN_LDS(lds);
    const bf16_t *kb = (const bf16_t *)a.k, *vb = (const bf16_t *)a.v;
    if constexpr (PAGED) { kb += kvh * a.head_stride; vb += kvh * a.head_stride; }
    else { kb += (long long)r0 * a.k_stride + kvh * HD; vb += (long long)r0 * a.v_stride + kvh * HD; }
    const const_ints table = (const_ints)(uintptr_t)(a.table + (PAGED ? (size_t)r * a.width : 0));

    // first row of the wavefront's i-th load of block c (rows past the request's last repeat that one)
    auto load_row = [&](int c, int i) { return min(c * BT_CH + (i * 4 + wave) * ROWS, last & -ROWS); };
    const int kpiece = (lane % SL) ^ ((wave * ROWS + lane / SL) & (SL - 1)), vpiece = (lane % SL) ^ (((lane / SL) & 3) << 1);
    int page[NI];
    auto look_up = [&](int c) {                               // the pages of block c
        if constexpr (PAGED)
#pragma unroll
            for (int i = 0; i < NI; ++i) page[i] = table[load_row(c, i) >> a.shift];
    };
    auto issue = [&](int c, int buf) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int b = load_row(c, i), in = min(lane / SL, last - b);
            const unsigned int d = l0 + buf * 2 * KV + (i * 4 + wave) * 1024;
            if constexpr (PAGED) {
                const int pg = (unsigned)page[i] < (unsigned)a.n_pages ? page[i] : 0;
                const long long at = pg * a.page_stride + (b & ((1 << a.shift) - 1)) * a.pos_stride;
                const unsigned int off = (unsigned int)in * (unsigned int)a.pos_stride * 2u;
                battn_dma(kb + at, off + kpiece * 16, d);
                battn_dma(vb + at, off + vpiece * 16, d + KV);
            } else {
                battn_dma(kb + b * a.k_stride, (unsigned int)in * (unsigned int)a.k_stride * 2u + kpiece * 16, d);
                battn_dma(vb + b * a.v_stride, (unsigned int)in * (unsigned int)a.v_stride * 2u + vpiece * 16, d + KV);
            }
        }
    };
    if (n_blocks > 0) {
        look_up(0);
        issue(0, 0);
        look_up(1);
    }
    bf16x8_t qf[KS];                                          // dimensions 16 ks + 8 half ... of the lane's pair
    {
        const bf16_t *qp = (const bf16_t *)a.q + (long long)(r0 + row) * a.q_stride + (kvh * a.group + g) * HD + half * 8;
        const unsigned int flip = a.scale2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(qp + ks * 16) ^ flip);
    }
    const float c2 = fabsf(a.scale2);
    float m = -INFINITY, off = -INFINITY, l = 0.f;
    f32x16_t o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    const int k_at = col * RB, v_row = 4 * half + ((lane & 15) >> 2), v_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);

    for (int c = 0; c < n_blocks; ++c) {
        const int buf = c & 1;
        battn_wait<0>();
        battn_meet();                                         // block c is here and nobody reads block c-1 any more
        if (c + 1 < n_blocks) {
            issue(c + 1, buf ^ 1);
            look_up(c + 2);
        }
        if (c * BT_CH > base + wave_last) continue;           // beyond all of the wavefront's rows
        const char *kl = lds + buf * 2 * KV;
        const unsigned int vl = l0 + buf * 2 * KV + KV;
        f32x16_t s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>(kl + t * 32 * RB + k_at + (((2 * ks + half) ^ (col & (SL - 1))) * 16)));
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[t], 0, 0, 0);
            }
        }
        const bool diagonal = c * BT_CH + BT_CH - 1 > base + wave_first;
        if (diagonal) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (c * BT_CH + t * 32 + 8 * (i / 4) + 4 * half + i % 4 > limit) s[t][i] = -INFINITY;
        }
        float cm = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) cm = fmaxf(cm, s[t][i]);
        cm = fmaxf(cm, lane_xor(cm, 32));
        m = fmaxf(m, cm);
        const float off_new = m == -INFINITY ? 0.f : battn_rounded_product(m, c2), f = __builtin_amdgcn_exp2f(off - off_new);
        off = off_new;
        float ps = 0.f;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], c2, -off));
                if (diagonal && c * BT_CH + t * 32 + 8 * (i / 4) + 4 * half + i % 4 > limit) s[t][i] = 0.f;      // (also where the scale is 0)
                ps += s[t][i];
            }
        l = l * f + ps;
        if (__any(f != 1.0f)) {
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= f;
        }
#pragma unroll
        for (int st = 0; st < 4; ++st) {                      // 16 positions
            const int t = st >> 1, i0 = (st & 1) * 8;
            const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, u32x4_t{pack_bf16(s[t][i0], s[t][i0 + 1]), pack_bf16(s[t][i0 + 2], s[t][i0 + 3]),
                                                                     pack_bf16(s[t][i0 + 4], s[t][i0 + 5]), pack_bf16(s[t][i0 + 6], s[t][i0 + 7])});
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                // (rows st*16 + v_row and 8 on: the row's number ends in v_row & 3, whatever st)
                const unsigned int at = vl + (st * 16 + v_row) * RB + (((4 * dt + (v_col >> 3)) ^ ((v_row & 3) << 1)) * 16) + (v_col & 4) * 2;
                const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(uintptr_t)at);
                const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(uintptr_t)(at + 8 * RB));
                const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb, o[dt], 0, 0, 0);
            }
        }
    }
    l += lane_xor(l, 32);
    if (live) {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        bf16_t *op = (bf16_t *)a.out + (long long)(r0 + row) * a.out_stride + (kvh * a.group + g) * HD + 4 * half;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const float v[4] = {o[t][4 * b] * inv, o[t][4 * b + 1] * inv, o[t][4 * b + 2] * inv, o[t][4 * b + 3] * inv};
                store_values<4>(op + t * 32 + b * 8, v);
            }
    }
}

// ------------------------------------------------------------------------------------------
// Few rows over a bf16 cache: what bounds them is the cache, read once. A request's (row, head) pairs of one kv head, 16 NT at a time, against
// all of its positions are a group; a group's blocks of 32 (heads of 64: 64) positions are units, and the units of the whole batch, group behind
// group, are dealt to the workgroups in equal runs (worked out by each for itself from the lengths). The four wavefronts of a workgroup take the
// blocks of a run in turn, keys and values straight from the cache to registers as operands, and are merged in LDS where a group ends. A
// group that lies in several runs leaves a partial result per run in the workspace; battn_merge_kernel joins them, in the order of the runs.
// As in the tile kernel everything is transposed, here in 16 x 16 tiles. Values are regrouped by byte permutes: a lane takes HD/16 neighbouring
// dimensions of its eight positions, so that matrix instruction t yields dimensions {HD/16 n + t}.
// NP = 3: fp32 queries, which stay exact as three bf16 planes, as do the weights.
// ------------------------------------------------------------------------------------------
constexpr int BF_WGS = 512;                                   // two workgroups per compute unit: 128 KB of the cache in flight on each
constexpr int BF_PAD = 4;                                     // floats behind a pair's HD values: its exponent, its sum

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// positions of a unit: 8 KB of keys, 8 KB of values, which a wavefront holds in registers
template <int HD> __host__ __device__ constexpr int battn_few_positions() { return 32 * 128 / HD; }
template <int HD> __host__ __device__ constexpr size_t battn_few_slot(int pairs) { return (size_t)pairs * (HD + BF_PAD); }      // floats of a partial result
// a group that begins in a run and does not end there: the runs that hold it, its first row's request, kv head, first pair and pairs
struct FewMerge { int runs, r0, kvh, pair, pairs; };
__host__ __device__ constexpr size_t battn_few_merges() { return BF_WGS * 32; }
static_assert(sizeof(FewMerge) <= 32, "");

// eight fp32 values as NP bf16 operands: rounded to nearest (1), or cut three times into exact parts (3)
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

// lane i's value, known to be the same everywhere (scalar registers, scalar loads)
__device__ __forceinline__ long long battn_lane(long long v, int i) {
    return (long long)(unsigned int)__builtin_amdgcn_readlane((int)v, i) | (long long)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32;
}

// x / d for 0 <= x < 2^53 and d > 0: many times shorter than a division of 64-bit integers
__device__ __forceinline__ long long battn_divide(long long x, long long d) {
    long long q = (long long)((double)x / (double)d);
    if (q * d > x) --q;
    if ((q + 1) * d <= x) ++q;
    return q;
}

// run that has a unit, where the first rem runs have q + 1 units and the others q
__device__ __forceinline__ int battn_run_of(long long unit, long long q, long long rem) {
    const long long longer = rem * (q + 1);
    return (int)(unit < longer ? battn_divide(unit, q + 1) : rem + battn_divide(unit - longer, q));
}

// units of request r: rows (0: not this kernel's), blocks of a group, groups of pairs per kv head
struct FewShape { int n, blocks, pair_groups; };
__device__ __forceinline__ FewShape battn_few_shape(const BattnArgs &a, int r, int group_pairs, int positions) {
    FewShape f{0, 1, 0};
    const int n = min(a.row_start[r + 1], a.n_rows) - max(a.row_start[r], 0);
    if (n > 0 && n <= a.few_rows) {
        f.n = n;
        f.blocks = max(1, (battn_len(a, r) + positions - 1) / positions);
        f.pair_groups = (int)(((long long)n * a.group + group_pairs - 1) / group_pairs);
    }
    return f;
}

template <int HD, int NT, int PW, int NP>
__host__ __device__ constexpr int battn_few_lds() {
    // the queries of a group [plane][pair][HD + 8] in bf16, and the wavefronts' shares [4][16][HD + BF_PAD] of one tile
    return NP * PW * NT * 16 * (HD + 8) * 2 + 4 * 16 * (HD + BF_PAD) * 4;
}

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

// PW: most wavefronts that share a block, where the pairs are more than one holds
template <int HD, int NT, int PW, int NP>
__global__ __launch_bounds__(256, 2) void battn_few_kernel(BattnArgs a) {
    constexpr int QS = HD / 32, DT = HD / 16, QROW = HD + 8, MROW = HD + BF_PAD, PAIRS = 16 * NT * PW, CH = battn_few_positions<HD>(), PT = CH / 16;
    typedef unsigned int vword __attribute__((ext_vector_type(DT / 2)));
    extern __shared__ __align__(16) char lds[];
    bf16_t *ql = (bf16_t *)lds;
    float *mb = (float *)(lds + NP * PAIRS * QROW * 2);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = lane >> 4, n16 = lane & 15;
    float *slots = (float *)((char *)a.ws + battn_few_merges());
    FewMerge *merges = (FewMerge *)a.ws;

    // All units, the first of this workgroup's run, and the request that has it: how many units lie before that one's. Up to 64 requests are looked at once.
    long long total = 0, before = 0, unit = 0, unit_end = 0, q = 0, rem = 0;
    int r = 0, runs = 0;
    const int w = blockIdx.x;
    if (tid == 0) merges[w] = FewMerge{0, 0, 0, 0, 0};
    auto run_start = [&](int i) { return i * q + min((long long)i, rem); };      // rem runs of q + 1 units, the others of q
    for (int pass = 0; pass < 2; ++pass) {
        bool found = false;
        for (int r0 = 0; r0 < a.n_requests && !found; r0 += 64) {
            long long upto = 0;
            if (r0 + lane < a.n_requests) {
                const FewShape g = battn_few_shape(a, r0 + lane, PAIRS, CH);
                upto = (long long)g.blocks * g.pair_groups * a.Hkv;
            }
            for (int off = 1; off < 64; off <<= 1) {
                const long long u = __shfl_up(upto, off);
                if (lane >= off) upto += u;
            }
            if (pass == 0) total += battn_lane(upto, 63);
            if (pass == 0 && r0 + 64 >= a.n_requests) {       // the total is known
                runs = (int)min((long long)gridDim.x, (total + 3) / 4);         // four units at least: a block for every wavefront
                if (w >= runs) return;
                q = battn_divide(total, runs);
                rem = total - q * runs;
                unit = run_start(w);
                unit_end = run_start(w + 1);
            }
            if (pass == 1 || a.n_requests <= 64) {
                const unsigned long long past = __ballot(unit < before + upto);
                found = past != 0;
                if (found) {
                    const int src = __builtin_ctzll(past);
                    r = r0 + src;
                    if (src > 0) before += battn_lane(upto, src - 1);
                } else {
                    before += battn_lane(upto, 63);
                }
            }
        }
        if (found) break;
    }
    const float c2 = fabsf(a.scale2);
    const unsigned int flip = a.scale2 < 0.f ? 0x80000000u : 0u;

    // Where the run is: a group, its blocks [b0, b1) of the run. What follows sets these for the blocks from `unit` on, and requests the group's
    // queries and the wavefront's first block.
    FewShape f = battn_few_shape(a, r, PAIRS, CH);
    int kvh, pg, b0, b1, r0, len, last, pairs, wp, wb, step, wave_pair;
    bool any;
    const_ints table;
    const bf16_t *kb, *vb;
    u32x4_t kf[PT][QS];                                       // position 16 pt + n16, dimensions 32 ks + 8 kg ...
    vword vr[PT][4];                                          // position 16 pt + 4 kg + i, dimensions DT n16 ...
    int page[PT][2];
    constexpr int NQ = (PAIRS * (HD / 8) + 255) / 256;        // 8 values of a query each: a thread's
    u32x4_t qv[NQ][NP == 1 ? 1 : 2];
    // first position of the block's e-th eight of tile pt (a page holds at least eight); positions past the last one repeat it
    auto eight = [&](int b, int pt, int e) __attribute__((always_inline)) { return min(b * CH + pt * 16 + e * 8, last & -8); };
    auto look_up = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int e = 0; e < 2; ++e) page[pt][e] = table[eight(b, pt, e) >> a.shift];
    };
    auto offset = [&](int b, int pt, int e) __attribute__((always_inline)) {
        const int id = __builtin_amdgcn_readfirstlane(page[pt][e]);      // (or a lane's choice between two becomes an index into memory)
        return ((unsigned)id < (unsigned)a.n_pages ? id : 0) * a.page_stride + (eight(b, pt, e) & ((1 << a.shift) - 1)) * a.pos_stride;
    };
    auto load_keys = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
            const long long lo = offset(b, pt, 0), hi = offset(b, pt, 1);
            const int in8 = min(n16 & 7, last - (n16 & 8 ? eight(b, pt, 1) : eight(b, pt, 0)));
            const bf16_t *kp = kb + (n16 & 8 ? hi : lo) + in8 * a.pos_stride + kg * 8;
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) kf[pt][ks] = *reinterpret_cast<const u32x4_t *>(kp + ks * 32);
        }
    };
    auto load_values = [&](int b) __attribute__((always_inline)) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
            const long long lo = offset(b, pt, 0), hi = offset(b, pt, 1);
            const int rest = last - (kg & 2 ? eight(b, pt, 1) : eight(b, pt, 0));
            const bf16_t *vp = vb + (kg & 2 ? hi : lo) + n16 * DT;
#pragma unroll
            for (int i = 0; i < 4; ++i) vr[pt][i] = *reinterpret_cast<const vword *>(vp + min((kg & 1) * 4 + i, rest) * a.pos_stride);
        }
    };
    auto enter = [&]() __attribute__((always_inline)) {
        while (unit - before >= (long long)f.blocks * f.pair_groups * a.Hkv && r + 1 < a.n_requests) {   // on to the next request with units
            before += (long long)f.blocks * f.pair_groups * a.Hkv;
            f = battn_few_shape(a, ++r, PAIRS, CH);
        }
        const long long in = unit - before;
        const int group = (int)battn_divide(in, f.blocks);
        b0 = (int)(in - (long long)group * f.blocks);
        b1 = (int)min((long long)f.blocks, b0 + (unit_end - unit));
        kvh = group / f.pair_groups;
        pg = group - kvh * f.pair_groups;
        r0 = max(a.row_start[r], 0);
        len = battn_len(a, r);
        last = len - 1;
        pairs = min(PAIRS, f.n * a.group - pg * PAIRS);       // (rows times heads: at most those of a call)
        // wavefronts that share a block, 16 NT pairs each; a wavefront's pairs; its blocks: wb, wb + step, ...
        const int pw = PW == 1 || pairs <= 16 * NT ? 1 : PW;
        wp = wave & (pw - 1); wb = wave / pw; step = 4 / pw; wave_pair = wp * 16 * NT;
        table = (const_ints)(uintptr_t)(a.table + (size_t)r * a.width);
        kb = (const bf16_t *)a.k + kvh * a.head_stride;
        vb = (const bf16_t *)a.v + kvh * a.head_stride;
        any = len > 0 && wave_pair < pairs && b0 + wb < b1;
        if (any) look_up(b0 + wb);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int p = (i * 256 + tid) / (HD / 8), d = (tid % (HD / 8)) * 8, pair = pg * PAIRS + min(p, pairs - 1);
            const long long at = (long long)(r0 + pair / a.group) * a.q_stride + (kvh * a.group + pair % a.group) * HD + d;
            if constexpr (NP == 1) {
                qv[i][0] = *reinterpret_cast<const u32x4_t *>((const bf16_t *)a.q + at);
            } else {
                qv[i][0] = *reinterpret_cast<const u32x4_t *>((const float *)a.q + at);
                qv[i][1] = *reinterpret_cast<const u32x4_t *>((const float *)a.q + at + 4);
            }
        }
        if (any) {
            load_keys(b0 + wb);
            load_values(b0 + wb);
            look_up(b0 + wb + step);
        }
    };
    enter();
    while (true) {
        const int base = len - f.n, pw = 4 / step;
        __syncthreads();                                      // nobody reads the last group's queries any more
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (PAIRS * (HD / 8) < 256 && tid >= PAIRS * (HD / 8)) break;
            bf16_t *to = ql + ((i * 256 + tid) / (HD / 8)) * QROW + (tid % (HD / 8)) * 8;
            if constexpr (NP == 1) {
                *reinterpret_cast<u32x4_t *>(to) = qv[i][0] ^ (flip | flip >> 16);
            } else {
                float v[8];
                bf16x8_t planes[3];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(qv[i][e >> 2][e & 3] ^ flip);
                battn_planes<3>(v, planes);
#pragma unroll
                for (int x = 0; x < 3; ++x) *reinterpret_cast<bf16x8_t *>(to + x * PAIRS * QROW) = planes[x];
            }
        }
        __syncthreads();

        int limit[NT];                                        // a pair's last visible position
        float off[NT], l[NT];
        f32x4_t o[NT][DT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            limit[t] = base + (pg * PAIRS + min(wave_pair + t * 16 + n16, pairs - 1)) / a.group;
            off[t] = -INFINITY;
            l[t] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        const int first_limit = base + pg * PAIRS / a.group;
        // (two builds, with a next block and without: what is in flight where a value is waited for has to be known)
        auto work = [&](int b, auto more_) __attribute__((always_inline)) {
            constexpr bool more = decltype(more_)::value;
            const int pos0 = b * CH;
            const bool diagonal = pos0 + CH - 1 > first_limit;
            f32x4_t s[NT][PT];
            const bf16_t *qb = ql + (wave_pair + n16) * QROW + kg * 8;
            if (NT * NP > 1) asm volatile("" : "+v"(qb));     // (they are read again for every block: there is no room to keep them all)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int pt = 0; pt < PT; ++pt) s[t][pt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                // the lowest plane first
#pragma unroll
                for (int q = NP - 1; q >= 0; --q)
#pragma unroll
                    for (int ks = 0; ks < QS; ++ks) {
                        const bf16x8_t qf = *reinterpret_cast<const bf16x8_t *>(qb + (q * PAIRS + t * 16) * QROW + ks * 32);
#pragma unroll
                        for (int pt = 0; pt < PT; ++pt) s[t][pt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[pt][ks]), qf, s[t][pt], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) load_keys(b + step);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (diagonal) {
#pragma unroll
                    for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (pos0 + pt * 16 + 4 * kg + i > limit[t]) s[t][pt][i] = -INFINITY;
                }
                float cm = s[t][0][0];
#pragma unroll
                for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) cm = fmaxf(cm, s[t][pt][i]);
                cm = fmaxf(cm, lane_xor(cm, 16));
                cm = fmaxf(cm, lane_xor(cm, 32));
                // (-inf times a scale of 0 would be NaN)
                const float off_new = cm == -INFINITY ? off[t] : fmaxf(off[t], battn_rounded_product(cm, c2)), ref = off_new == -INFINITY ? 0.f : off_new;
                const float fac = __builtin_amdgcn_exp2f(off[t] - ref);
                off[t] = off_new;
                float ps = 0.f;
#pragma unroll
                for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[t][pt][i] = __builtin_amdgcn_exp2f(fmaf(s[t][pt][i], c2, -ref));
                        if (diagonal && pos0 + pt * 16 + 4 * kg + i > limit[t]) s[t][pt][i] = 0.f;
                        ps += s[t][pt][i];
                    }
                l[t] = l[t] * fac + ps;
                if (__any(fac != 1.0f)) {
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[t][d] *= fac;
                }
            }
            u32x4_t vf[PT / 2][DT];                           // the values' operands: positions 2j, 2j+1 of the lane's eight
#pragma unroll
            for (int hf = 0; hf < PT / 2; ++hf)
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        vf[hf][d][j] = __builtin_amdgcn_perm(vr[2 * hf + (j >> 1)][2 * (j & 1) + 1][d >> 1], vr[2 * hf + (j >> 1)][2 * (j & 1)][d >> 1],
                                                             (d & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int hf = 0; hf < PT / 2; ++hf)
#pragma unroll
                for (int d = 0; d < DT; ++d) asm volatile("" : "+v"(vf[hf][d]));       // all of it here: the next values go to the same registers
            if constexpr (more) {
                load_values(b + step);
                look_up(b + 2 * step);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int hf = 0; hf < PT / 2; ++hf) {
                    const f32x4_t x = s[t][2 * hf], y = s[t][2 * hf + 1];
                    const float pv[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                    bf16x8_t pb[NP];
                    battn_planes<NP>(pv, pb);
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int q = NP - 1; q >= 0; --q)
                            o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf[hf][d]), pb[q], o[t][d], 0, 0, 0);
                }
        };
        if (any) {
            int b = b0 + wb;
            for (; b + step < b1; b += step) work(b, std::true_type{});
            work(b, std::false_type{});
        }

        // the run goes on: the next group's loads are on their way while this one is finished
        const bool whole = b0 == 0 && b1 == f.blocks, begins = b0 == 0, goes_on = unit + (b1 - b0) < unit_end;
        const int this_pairs = pairs, this_r0 = r0, this_kvh = kvh, this_pair = pg * PAIRS;
        const long long group_end = unit - b0 + f.blocks - 1;     // the group's last unit
        unit += b1 - b0;
        if (goes_on) enter();

        // the wavefronts' shares of each tile: thread (pair, dimensions) adds them up and writes them out, or leaves them for the merge
        float *slot = slots + (size_t)(2 * w + begins) * battn_few_slot<HD>(PAIRS);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            l[t] += lane_xor(l[t], 16);
            l[t] += lane_xor(l[t], 32);
            float *mine = mb + (wave * 16 + n16) * MROW;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int d = 0; d < DT; d += 4)
                    *reinterpret_cast<f32x4_t *>(mine + DT * (4 * kg + q) + d) = f32x4_t{o[t][d][q], o[t][d + 1][q], o[t][d + 2][q], o[t][d + 3][q]};
            if (kg == 0) { mine[HD] = off[t]; mine[HD + 1] = l[t]; }
            __syncthreads();
            constexpr int V = HD * PW / 16, TP = HD / V;      // values per thread, threads per pair
            const int q16 = tid / TP, p = (q16 >> 4) * 16 * NT + t * 16 + (q16 & 15), d0 = (tid % TP) * V;
            const float *share = mb + (((q16 >> 4) & (pw - 1)) * 16 + (q16 & 15)) * MROW;         // of the first of the wavefronts that have this pair
            float top = -INFINITY, sum = 0.f, v[V];
            for (int x = 0; x < 4; x += pw) top = fmaxf(top, share[x * 16 * MROW + HD]);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = 0.f;
            for (int x = 0; x < 4; x += pw) {
                const float *m = share + x * 16 * MROW;
                const float k = m[HD] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[HD] - top);
                sum = fmaf(m[HD + 1], k, sum);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = fmaf(m[d0 + e], k, v[e]);
            }
            if (p < this_pairs && q16 < 16 * pw) {
                if (whole) {
                    battn_few_out<V, HD, NP>(a, this_r0, this_kvh, this_pair + p, d0, v, sum);
                } else {
                    float *to = slot + p * MROW;
                    store_values<V>(to + d0, v);
                    if (d0 == 0) { to[HD] = top; to[HD + 1] = sum; }
                }
            }
            __syncthreads();
        }
        if (!whole && begins && tid == 0)                     // it goes on in the runs behind this one
            merges[w] = FewMerge{battn_run_of(group_end, q, rem) - w + 1, this_r0, this_kvh, this_pair, this_pairs};
        if (!goes_on) return;
    }
}

// Joins the partial results of a group. HD/4 lanes have a pair, four values each, and take its runs' results one after the other, four requested at a
// time; where the group lies in more than four runs, four such teams share them. In a launch of its own: the last workgroup of a group doing it inside
// the first launch had to fetch up to 32 runs' results of all pairs by itself, one memory latency after the other (two requests at
// 100 000 positions: 286 us in all, 168 us in two launches).
constexpr int BM_NT = 256;
template <int HD> __host__ __device__ constexpr int battn_merge_teams() { return BM_NT * 4 / HD; }
template <int HD, int NP>
__global__ __launch_bounds__(BM_NT) void battn_merge_kernel(BattnArgs a, int slot_pairs) {
    constexpr int LP = HD / 4, TEAMS = battn_merge_teams<HD>(), MROW = HD + BF_PAD, U = 4;
    __shared__ f32x4_t part[TEAMS][LP];
    __shared__ float part_top[TEAMS], part_sum[TEAMS];
    const FewMerge m = ((const FewMerge *)a.ws)[blockIdx.x];
    if (m.runs == 0) return;                                  // the whole workgroup
    const int lane = threadIdx.x % LP, team = threadIdx.x / LP;
    const int subs = m.runs > 4 ? 4 : 1, sub = team & (subs - 1), at_once = TEAMS / subs;
    const size_t slot = battn_few_slot<HD>(slot_pairs);
    for (int p0 = blockIdx.y * at_once; p0 < m.pairs; p0 += gridDim.y * at_once) {
        const int p = p0 + team / subs;
        // run x's partial result is its second one (a group that begins there) for the first run, its first one for the others
        const float *first = (const float *)((const char *)a.ws + battn_few_merges()) + 2 * blockIdx.x * slot + min(p, m.pairs - 1) * MROW;
        float top = -INFINITY, sum = 0.f;
        f32x4_t v{0.f, 0.f, 0.f, 0.f};
        for (int x = sub; x < m.runs; x += subs * U) {
            float at[U], l[U];
            f32x4_t w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int y = x + subs * u;
                at[u] = -INFINITY;
                if (y < m.runs) {
                    const float *from = first + (2 * y + (y == 0)) * slot;
                    at[u] = from[HD];
                    l[u] = from[HD + 1];
                    w[u] = *reinterpret_cast<const f32x4_t *>(from + lane * 4);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (at[u] == -INFINITY) continue;
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
