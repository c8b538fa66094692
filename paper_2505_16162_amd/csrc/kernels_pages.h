// Pages of a batch of requests: who holds which (page_plan_kernel), where a round's rows go (page_rows_kernel), and the rotary
// embedding and cache write of those rows (paged_store_kernel).
#pragma once
#include "device_ops.h"

namespace ks {

constexpr int PLAN_MAX_REQUESTS = 4096;                       // what the plan keeps in LDS
constexpr int PLAN_ROWS_NT = 256;
constexpr int PLAN_U = 4;                                     // pages a thread has under way

struct PlanArgs {
    int *table, *held, *free_pages, *n_free;
    const int *cached, *added;
    int *row_start, *kv_len, *slots, *positions, *result;
    int n, width, n_pages, shift;                             // page size = 1 << shift
    int max_rows;
    int rows_here;                                            // 1: the plan's own workgroup fills in slots and positions
};

// last entry of at[0..n] (ascending, at[0] = 0) that is not above k < at[n]
__device__ __forceinline__ int plan_owner(const int *at, int n, int k) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= k) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void plan_row(const PlanArgs &a, const int *row_at, int t) {
    int slot = -1, pos = -1;
    if (t < row_at[a.n]) {
        const int r = plan_owner(row_at, a.n, t);
        pos = a.kv_len[r] + (t - row_at[r + 1]);
        slot = (a.table[(size_t)r * a.width + (pos >> a.shift)] << a.shift) + (pos & ((1 << a.shift) - 1));
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
}

// One workgroup. Per request the pages it needs, gives back and takes; three prefix sums (rows, pages back, pages taken) turn
// the stack into arithmetic: the k-th page given back (ascending) is pushed to n_free + n_back - 1 - k, the k-th page taken is popped
// from n_free + n_back - 1 - k, whatever it was (the stack is read and written at computed places: no page waits for another). Bound by latency, a
// chain of a dozen dependent steps. Nothing is changed before the totals have shown that all of it can be done, and no cached or added length is read
// after the first result has been written: either may be the array that the new lengths go to.
template <int PLAN_NT, int PLAN_PER>
__global__ __launch_bounds__(PLAN_NT) void page_plan_kernel(PlanArgs a) {
    constexpr int MOST = PLAN_NT * PLAN_PER;
    __shared__ int row_at[MOST + 1], back_at[MOST + 1], take_at[MOST + 1];
    __shared__ long long wave_sums[PLAN_NT / 64][3];
    __shared__ int wave_max[PLAN_NT / 64], wave_bad[PLAN_NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const long long page = 1ll << a.shift;
    const int n_free = *a.n_free;
    int bad = (n_free < 0 || n_free > a.n_pages) ? 1 : 0, longest = 0;
    long long rows[PLAN_PER], back[PLAN_PER], take[PLAN_PER], len[PLAN_PER], s[3] = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = tid * PLAN_PER + i;
        rows[i] = back[i] = take[i] = len[i] = 0;
        if (r < a.n) {
            const long long c = a.cached[r], d = a.added[r], held = a.held[r], need = (c + d + page - 1) >> a.shift;
            len[i] = c + d;
            if (c < 0 || d < 0 || len[i] > 0x7fffffffll || held < 0 || held > a.width) bad |= 1;
            if (need > a.width) bad |= 4;
            rows[i] = d;
            back[i] = held > need ? held - need : 0;
            take[i] = need > held ? need - held : 0;
            longest = max(longest, (int)len[i]);
        }
        s[0] += rows[i]; s[1] += back[i]; s[2] += take[i];
    }
    // prefix sums over the threads
    long long before[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        long long v = s[q];
        for (int off = 1; off < 64; off <<= 1) {
            const long long u = __shfl_up(v, off);
            if (lane >= off) v += u;
        }
        before[q] = v - s[q];
        if (lane == 63) wave_sums[wave][q] = v;
    }
    for (int off = 32; off; off >>= 1) {
        bad |= __shfl_xor(bad, off);
        longest = max(longest, __shfl_xor(longest, off));
    }
    if (lane == 0) { wave_max[wave] = longest; wave_bad[wave] = bad; }
    __syncthreads();
    // the same over the wavefronts, a lane each
    constexpr int NW = PLAN_NT / 64;
    long long total[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const long long own = wave_sums[lane % NW][q];
        long long v = own;
#pragma unroll
        for (int off = 1; off < NW; off <<= 1) {
            const long long u = __shfl_up(v, off, NW);
            if (lane % NW >= off) v += u;
        }
        before[q] += __shfl(v - own, wave);
        total[q] = __shfl(v, NW - 1);
    }
    bad |= wave_bad[lane % NW];
    longest = max(longest, wave_max[lane % NW]);
#pragma unroll
    for (int off = 1; off < NW; off <<= 1) {
        bad |= __shfl_xor(bad, off);
        longest = max(longest, __shfl_xor(longest, off));
    }
    if (n_free + total[1] > a.n_pages) bad |= 1;
    if (total[0] > a.max_rows) bad |= 2;
    if (total[2] > n_free + total[1]) bad |= 8;
    if (bad) {
        const int flag = (bad & 1) ? 1 : (bad & 2) ? 2 : (bad & 4) ? 3 : 4;
        for (int r = tid; r <= a.n; r += PLAN_NT) {
            a.row_start[r] = 0;
            if (r < a.n) a.kv_len[r] = 0;
        }
        if (a.rows_here)
            for (int t = tid; t < a.max_rows; t += PLAN_NT) { a.slots[t] = -1; a.positions[t] = -1; }
        if (tid == 0) { a.result[0] = 0; a.result[1] = 0; a.result[2] = flag; a.result[3] = 0; }
        return;
    }
    const int n_back = (int)total[1], n_take = (int)total[2], top = n_free + n_back;      // (at most the pool's and the tables' sizes)
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = tid * PLAN_PER + i;
        if (r <= a.n) {
            row_at[r] = (int)before[0]; back_at[r] = (int)before[1]; take_at[r] = (int)before[2];
            a.row_start[r] = (int)before[0];
            if (r < a.n) a.kv_len[r] = (int)(len[i]);
        }
        before[0] += rows[i]; before[1] += back[i]; before[2] += take[i];
    }
    if (tid == PLAN_NT - 1 && a.n == MOST) {
        row_at[a.n] = (int)total[0]; back_at[a.n] = n_back; take_at[a.n] = n_take;
        a.row_start[a.n] = (int)total[0];
    }
    __syncthreads();
    for (int k0 = tid; k0 < n_back; k0 += PLAN_U * PLAN_NT) {
        int *entry[PLAN_U], page_id[PLAN_U];
#pragma unroll
        for (int u = 0; u < PLAN_U; ++u) {
            const int k = min(k0 + u * PLAN_NT, n_back - 1), r = plan_owner(back_at, a.n, k);
            const int need = (int)((a.kv_len[r] + page - 1) >> a.shift);
            entry[u] = a.table + (size_t)r * a.width + need + (k - back_at[r]);
            page_id[u] = *entry[u];
        }
#pragma unroll
        for (int u = 0; u < PLAN_U; ++u)
            if (k0 + u * PLAN_NT < n_back) {
                a.free_pages[top - 1 - (k0 + u * PLAN_NT)] = page_id[u];
                *entry[u] = -1;
            }
    }
    __syncthreads();
    for (int k0 = tid; k0 < n_take; k0 += PLAN_U * PLAN_NT) {
        int *entry[PLAN_U], page_id[PLAN_U];
#pragma unroll
        for (int u = 0; u < PLAN_U; ++u) {
            const int k = min(k0 + u * PLAN_NT, n_take - 1), r = plan_owner(take_at, a.n, k);
            entry[u] = a.table + (size_t)r * a.width + a.held[r] + (k - take_at[r]);
            page_id[u] = a.free_pages[top - 1 - k];
        }
#pragma unroll
        for (int u = 0; u < PLAN_U; ++u)
            if (k0 + u * PLAN_NT < n_take) {
                *entry[u] = page_id[u];
                a.free_pages[top - 1 - (k0 + u * PLAN_NT)] = -1;
            }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PLAN_PER; ++i) {
        const int r = tid * PLAN_PER + i;
        if (r < a.n) a.held[r] = (int)((a.kv_len[r] + page - 1) >> a.shift);
    }
    if (tid == 0) {
        *a.n_free = top - n_take;
        a.result[0] = (int)total[0]; a.result[1] = n_take - n_back; a.result[2] = 0; a.result[3] = longest;
    }
    if (a.rows_here)
        for (int t = tid; t < a.max_rows; t += PLAN_NT) plan_row(a, row_at, t);
}

// slots and positions of many rows, behind the plan
__global__ __launch_bounds__(PLAN_ROWS_NT) void page_rows_kernel(PlanArgs a) {
    __shared__ int row_at[PLAN_MAX_REQUESTS + 1];
    for (int r = threadIdx.x; r <= a.n; r += PLAN_ROWS_NT) row_at[r] = a.row_start[r];
    __syncthreads();
    for (long long t = (long long)blockIdx.x * PLAN_ROWS_NT + threadIdx.x; t < a.max_rows; t += (long long)gridDim.x * PLAN_ROWS_NT) plan_row(a, row_at, (int)t);
}

// ------------------------------------------------------------------------------------------
// Rotary embedding and cache write. A workgroup takes one row and a range of its heads; a thread takes 16 bytes of a head's first half
// and the 16 bytes of the second half that they are paired with. The row's angles are the same for every head: 2^(-2i/hd log2 base) turns
// times the position in 64 bits, the whole turns taken off there, sine and cosine of the rest in fp32; one thread per
// pair works them out into LDS while the row's loads are under way. Bound by memory: 542 MB read and written in 107 us, 5.07 TB/s,
// what a copy of that size reaches.
// ------------------------------------------------------------------------------------------
struct StoreArgs {
    const void *qkv;
    void *q_out, *k_out, *k, *v;
    const int *slots, *positions;
    long long qkv_stride, q_stride, k_stride, page_stride, head_stride, pos_stride;
    int n_heads, n_kv, shift;
    int n_slots;                        // n_pages * page size
    double log2_base;
};

constexpr int STORE_NT = 256, STORE_U = 4;      // threads, pieces a thread has under way

template <typename T> struct Piece;             // 16 bytes of a row
template <> struct Piece<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void load(const float *p, float *v) {
        const float4 t = *reinterpret_cast<const float4 *>(p);
        v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
    }
};
template <> struct Piece<bf16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void load(const bf16_t *p, float *v) {
        const uint4 t = *reinterpret_cast<const uint4 *>(p);
        const unsigned int w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
// two values rounded to bf16 (nearest even, NaN stays NaN), packed
__device__ __forceinline__ unsigned int pack_bf16(float a, float b) {
    return __builtin_bit_cast(unsigned int, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}
template <int N> __device__ __forceinline__ void store_values(float *p, const float *v) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = float4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
template <int N> __device__ __forceinline__ void store_values(bf16_t *p, const float *v) {
    if constexpr (N >= 8) {
#pragma unroll
        for (int i = 0; i < N; i += 8)
            *reinterpret_cast<uint4 *>(p + i) = uint4{pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3]), pack_bf16(v[i + 4], v[i + 5]), pack_bf16(v[i + 6], v[i + 7])};
    } else {
        *reinterpret_cast<uint2 *>(p) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    }
}

template <int HD, typename T, typename KT>
__global__ __launch_bounds__(STORE_NT) void paged_store_kernel(StoreArgs a) {
    constexpr int N = Piece<T>::N, HALF = HD / 2, PER = HALF / N;         // values a piece, pieces of a head's half
    __shared__ float cos_t[HALF], sin_t[HALF];
    const int row = blockIdx.x, slot = a.slots[row], pos = a.positions[row];
    if ((unsigned)slot >= (unsigned)a.n_slots || pos < 0) return;        // the whole workgroup
    const int n_items = (a.n_heads + 2 * a.n_kv) * PER;
    const T *src = (const T *)a.qkv + row * a.qkv_stride;
    const int first = blockIdx.y * (STORE_NT * STORE_U) + threadIdx.x;
    float x[STORE_U][N], y[STORE_U][N];
#pragma unroll
    for (int u = 0; u < STORE_U; ++u) {
        const int i = first + u * STORE_NT;
        if (i < n_items) {
            const T *p = src + (i / PER) * HD + (i % PER) * N;
            Piece<T>::load(p, x[u]);
            Piece<T>::load(p + HALF, y[u]);
        }
    }
    if (threadIdx.x < HALF) {
        const double turns = (double)pos * (exp2((double)threadIdx.x * (-2.0 / HD) * a.log2_base) * 0.15915494309189533577);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        cos_t[threadIdx.x] = c;
        sin_t[threadIdx.x] = s;
    }
    __syncthreads();
    const long long at = (long long)(slot >> a.shift) * a.page_stride + (long long)(slot & ((1 << a.shift) - 1)) * a.pos_stride;
#pragma unroll
    for (int u = 0; u < STORE_U; ++u) {
        const int i = first + u * STORE_NT;
        if (i >= n_items) break;
        const int head = i / PER, d = (i % PER) * N;
        if (head < a.n_heads + a.n_kv) {
            float f[N], g[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float c = cos_t[d + e], s = sin_t[d + e];
                f[e] = x[u][e] * c - y[u][e] * s;
                g[e] = y[u][e] * c + x[u][e] * s;
            }
            T *rows = head < a.n_heads ? (T *)a.q_out : (T *)a.k_out;
            if (rows) {
                T *p = rows + row * (head < a.n_heads ? a.q_stride : a.k_stride) + (head < a.n_heads ? head : head - a.n_heads) * HD + d;
                store_values<N>(p, f);
                store_values<N>(p + HALF, g);
            }
            if (head >= a.n_heads) {
                KT *p = (KT *)a.k + at + (head - a.n_heads) * a.head_stride + d;
                store_values<N>(p, f);
                store_values<N>(p + HALF, g);
            }
        } else {
            KT *p = (KT *)a.v + at + (head - a.n_heads - a.n_kv) * a.head_stride + d;
            store_values<N>(p, x[u]);
            store_values<N>(p + HALF, y[u]);
        }
    }
}

}  // namespace ks
