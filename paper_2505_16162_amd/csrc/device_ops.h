// What the kernels of every source share: bf16 as it is stored, and exchanges and reductions over a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ks {

typedef uint16_t bf16_t;  // raw bit pattern

// ints that nothing writes while the kernel runs, by scalar loads where the index is the same for all lanes
typedef const __attribute__((address_space(4))) int *const_ints;

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

__device__ __forceinline__ float bf16_to_float(bf16_t b) { return __uint_as_float(((uint32_t)b) << 16); }

// fp32 -> bf16, round to nearest even (inf/nan pass through with the payload truncated)
__device__ __forceinline__ bf16_t float_to_bf16_rne(float f) {
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7f800000u) == 0x7f800000u) return (bf16_t)(u >> 16);
    u += 0x7fffu + ((u >> 16) & 1u);
    return (bf16_t)(u >> 16);
}

__device__ __forceinline__ float load_as_float(const float *p, size_t i) { return p[i]; }
__device__ __forceinline__ float load_as_float(const bf16_t *p, size_t i) { return bf16_to_float(p[i]); }
__device__ __forceinline__ void store_rounded(float *p, size_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store_rounded(bf16_t *p, size_t i, float v) { p[i] = float_to_bf16_rne(v); }

// The value of lane ^ off (off: 1, 2, 4, .. 32, a constant once the loop around it is unrolled) by the cross-lane moves of the
// vector ALU. __shfl_xor goes through the LDS unit instead: 64 and more cycles for each of the dependent exchanges of a
// reduction, where these take 4 to 8. The reductions add the same pairs in the same order either way. K-best search (200 000 x 5120,
// three queries): 466 -> 455 us, the two selection stages 25.5 + 21.0 -> 23.5 + 19.8 us; routing over a small table 22.8 -> 21.7 us.
template <int CTRL, int BANKS = 0xf>
__device__ __forceinline__ int lane_dpp(int old, int v) { return __builtin_amdgcn_update_dpp(old, v, CTRL, 0xf, BANKS, false); }
__device__ __forceinline__ int lane_xor(int v, int off) {
    switch (off) {
        case 1: return lane_dpp<0xb1>(v, v);                                // quad_perm 1 0 3 2
        case 2: return lane_dpp<0x4e>(v, v);                                // quad_perm 2 3 0 1
        case 4: return lane_dpp<0x114, 0xa>(lane_dpp<0x104, 0x5>(v, v), v); // even quads from the quad above, odd ones from the one below
        case 8: return lane_dpp<0x128>(v, v);                               // the row of 16 rotated by half
        case 16: {
            const auto r = __builtin_amdgcn_permlane16_swap((unsigned int)v, (unsigned int)v, false, false);
            return (int)((threadIdx.x & 16) ? r[0] : r[1]);
        }
        default: {
            const auto r = __builtin_amdgcn_permlane32_swap((unsigned int)v, (unsigned int)v, false, false);
            return (int)((threadIdx.x & 32) ? r[0] : r[1]);
        }
    }
}
__device__ __forceinline__ float lane_xor(float v, int off) { return __int_as_float(lane_xor(__float_as_int(v), off)); }

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += lane_xor(v, off);
    return v;
}
// the same sum with __shfl_xor, for the kernels whose loads are placed by hand: the lane exchanges above take register copies, which
// the build's check of those kernels does not tell from copies of a load in flight
__device__ __forceinline__ float wave_sum_shfl(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, lane_xor(v, off));
    return v;
}

}  // namespace ks
