// Attention of a batch's few rows over pages in bf16.
#pragma once
#include <cfloat>

#include "battn_common.h"

namespace ks {

// ------------------------------------------------------------------------------------------
// Few rows over a bf16 cache: what bounds them is the cache, read once. A request's (row, head) pairs of one kv head, 16 at a time, against
// all of its positions are a group; a group's blocks of 32 (heads of 64: 64) positions are units, and the units of the whole batch, group behind
// group, are dealt to the workgroups in equal runs (worked out by each for itself from the lengths). The four wavefronts of a workgroup take the
// blocks of a run in turn, keys and values straight from the cache to registers as operands, and are merged in LDS where a group ends. A
// group that lies in several runs leaves a partial result per run in the workspace; battn_merge_kernel joins them, in the order of the runs.
// As in the tile kernel everything is transposed, here in 16 x 16 tiles. Values are regrouped by byte permutes: a lane takes HD/16 neighbouring
// dimensions of its eight positions, so that matrix instruction t yields dimensions {HD/16 n + t}.
// NP = 3: fp32 queries, which stay exact as three bf16 planes, as do the weights.
// 12 requests of 2 to 5 rows, 40 kv heads of 128, fp32 queries: 413 MB in 84 us with the merge, 4.9 TB/s.
// ------------------------------------------------------------------------------------------

// positions of a unit: 8 KB of keys, 8 KB of values, which a wavefront holds in registers
template <int HD> __host__ __device__ constexpr int battn_few_positions() { return 32 * 128 / HD; }
// units of request r: rows, blocks of a group, groups of pairs per kv head
struct FewShape { int n, blocks, pair_groups; };
__device__ __forceinline__ FewShape battn_few_shape(const BattnArgs &a, int r, int group_pairs, int positions) {
    FewShape f{0, 1, 0};
    const int n = rows_of(a.row_start, r, a.n_rows).n;
    if (n > 0) {
        f.n = n;
        f.blocks = max(1, (battn_len(a, r) + positions - 1) / positions);
        f.pair_groups = (int)(((long long)n * a.group + group_pairs - 1) / group_pairs);
    }
    return f;
}

template <int HD, int NP>
__global__ __launch_bounds__(256, 2) void battn_few_kernel(BattnArgs a) {
    constexpr int QS = HD / 32, DT = HD / 16, MROW = HD + BF_PAD, PAIRS = 16, CH = battn_few_positions<HD>(), PT = CH / 16;
    typedef unsigned int vword __attribute__((ext_vector_type(DT / 2)));
    __shared__ __align__(16) float mb[4 * 16 * MROW];         // the wavefronts' shares of a group
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kg = lane >> 4, n16 = lane & 15;
    float *slots = (float *)((char *)a.ws + battn_few_merges());
    FewMerge *merges = (FewMerge *)a.ws;

    // All units, the first of this workgroup's run, and the request that has it: how many units lie before that one's. Up to 64 requests are looked at once.
    long long total = 0, before = 0, unit = 0, unit_end = 0, q = 0, rem = 0;
    int r = 0, runs = 0;
    const int w = battn_run();
    if (tid == 0) merges[w] = FewMerge{0, 0, 0, 0, 0};
    auto run_start = [&](int i) { return battn_same(i * q + min((long long)i, rem)); };      // rem runs of q + 1 units, the others of q
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
                runs = battn_same((int)min((long long)gridDim.x, (total + 3) / 4));         // four units at least: a block for every wavefront
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
    const float c2 = fmaxf(fabsf(a.scale2), FLT_MIN);         // (a hidden score, -inf, has to stay that under a scale of 0)
    const unsigned int flip = a.scale2 < 0.f ? 0x80000000u : 0u;

    // Where the run is: a group, its blocks [b0, b1) of the run. What follows sets these for the blocks from `unit` on, and requests the group's
    // queries and the wavefront's first block.
    FewShape f = battn_few_shape(a, r, PAIRS, CH);
    int kvh, pg, b0, b1, r0, len, last, pairs;
    bool any;
    const_ints table;
    const bf16_t *kb, *vb;
    u32x4_t kf[PT][QS];                                       // position 16 pt + n16, dimensions 32 ks + 8 kg ...
    vword vr[PT][4];                                          // position 16 pt + 4 kg + i, dimensions DT n16 ...
    int page[PT][2];
    u32x4_t qv[QS][NP == 1 ? 1 : 2];                          // the next group's queries: pair n16, dimensions 32 ks + 8 kg ...
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
    auto load_queries = [&]() __attribute__((always_inline)) {
        const int pair = pg * PAIRS + min(n16, pairs - 1);
        const long long at = (long long)(r0 + pair / a.group) * a.q_stride + (kvh * a.group + pair % a.group) * HD + kg * 8;
#pragma unroll
        for (int ks = 0; ks < QS; ++ks) {
            if constexpr (NP == 1) {
                qv[ks][0] = *reinterpret_cast<const u32x4_t *>((const bf16_t *)a.q + at + ks * 32);
            } else {
                qv[ks][0] = *reinterpret_cast<const u32x4_t *>((const float *)a.q + at + ks * 32);
                qv[ks][1] = *reinterpret_cast<const u32x4_t *>((const float *)a.q + at + ks * 32 + 4);
            }
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
        b1 = battn_same((int)min((long long)f.blocks, b0 + (unit_end - unit)));
        kvh = group / f.pair_groups;
        pg = group - kvh * f.pair_groups;
        r0 = rows_of(a.row_start, r, a.n_rows).first;
        len = battn_same(battn_len(a, r));
        last = len - 1;
        pairs = min(PAIRS, f.n * a.group - pg * PAIRS);       // (rows times heads: at most those of a call)
        table = a.table + (size_t)r * a.width;
        kb = (const bf16_t *)a.k + kvh * a.head_stride;
        vb = (const bf16_t *)a.v + kvh * a.head_stride;
        any = len > 0 && b0 + wave < b1;
        if (any) look_up(b0 + wave);
        if constexpr (NP == 1) load_queries();                // (there is no room for fp32 ones beside the last group's)
        if (any) {
            load_keys(b0 + wave);
            load_values(b0 + wave);
            look_up(b0 + wave + 4);
        }
    };
    enter();
    while (true) {
        const int base = len - f.n;
        const int limit = base + (pg * PAIRS + min(n16, pairs - 1)) / a.group, first_limit = base + pg * PAIRS / a.group;      // last visible position of the lane's pair, of the first
        bf16x8_t qf[QS][NP];
        if constexpr (NP == 3) load_queries();
#pragma unroll
        for (int ks = 0; ks < QS; ++ks) {
            if constexpr (NP == 1) {
                qf[ks][0] = __builtin_bit_cast(bf16x8_t, qv[ks][0] ^ (flip | flip >> 16));
            } else {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(qv[ks][e >> 2][e & 3] ^ flip);
                battn_planes<3>(v, qf[ks]);
            }
        }
        float off = -INFINITY, l = 0.f;
        f32x4_t o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        // (two builds, with a next block and without: what is in flight where a value is waited for has to be known)
        auto work = [&](int b, auto more_) __attribute__((always_inline)) {
            constexpr bool more = decltype(more_)::value;
            const int pos0 = b * CH;
            f32x4_t s[PT];
#pragma unroll
            for (int pt = 0; pt < PT; ++pt) s[pt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            // the lowest plane first
#pragma unroll
            for (int q = NP - 1; q >= 0; --q)
#pragma unroll
                for (int ks = 0; ks < QS; ++ks)
#pragma unroll
                    for (int pt = 0; pt < PT; ++pt) s[pt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[pt][ks]), qf[ks][q], s[pt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more) load_keys(b + 4);
            __builtin_amdgcn_sched_barrier(0);
            if (pos0 + CH - 1 > first_limit) {
#pragma unroll
                for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (pos0 + pt * 16 + 4 * kg + i > limit) s[pt][i] = -INFINITY;
            }
            float cm = s[0][0];
#pragma unroll
            for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                for (int i = 0; i < 4; ++i) cm = fmaxf(cm, s[pt][i]);
            cm = fmaxf(cm, lane_xor(cm, 16));
            cm = fmaxf(cm, lane_xor(cm, 32));
            const float off_new = fmaxf(off, battn_rounded_product(cm, c2)), ref = off_new == -INFINITY ? 0.f : off_new;
            const float fac = __builtin_amdgcn_exp2f(off - ref);
            off = off_new;
            float ps = 0.f;
#pragma unroll
            for (int pt = 0; pt < PT; ++pt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[pt][i] = __builtin_amdgcn_exp2f(fmaf(s[pt][i], c2, -ref));
                    ps += s[pt][i];
                }
            l = l * fac + ps;
            if (__any(fac != 1.0f)) {
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= fac;
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
                load_values(b + 4);
                look_up(b + 8);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int hf = 0; hf < PT / 2; ++hf) {
                const f32x4_t x = s[2 * hf], y = s[2 * hf + 1];
                const float pv[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                bf16x8_t pb[NP];
                battn_planes<NP>(pv, pb);
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int q = NP - 1; q >= 0; --q) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf[hf][d]), pb[q], o[d], 0, 0, 0);
            }
        };
        if (any) {
            int b = b0 + wave;
            for (; b + 4 < b1; b += 4) work(b, std::true_type{});
            work(b, std::false_type{});
        }

        // the run goes on: the next group's loads are on their way while this one is finished
        const bool whole = b0 == 0 && b1 == f.blocks, begins = b0 == 0, goes_on = unit + (b1 - b0) < unit_end;
        const int this_pairs = pairs, this_r0 = r0, this_kvh = kvh, this_pair = pg * PAIRS;
        const long long group_end = unit - b0 + f.blocks - 1;     // the group's last unit
        unit += b1 - b0;
        if (goes_on) enter();

        // the wavefronts' shares: thread (pair, dimensions) adds them up and writes them out, or leaves them for the merge
        l += lane_xor(l, 16);
        l += lane_xor(l, 32);
        float *mine = mb + (wave * 16 + n16) * MROW;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int d = 0; d < DT; d += 4) *reinterpret_cast<f32x4_t *>(mine + DT * (4 * kg + q) + d) = f32x4_t{o[d][q], o[d + 1][q], o[d + 2][q], o[d + 3][q]};
        if (kg == 0) { mine[HD] = off; mine[HD + 1] = l; }
        __syncthreads();
        constexpr int V = HD / 16;                            // values per thread
        const int p = tid >> 4, d0 = (tid & 15) * V;
        const float *share = mb + p * MROW;
        float top = -INFINITY, sum = 0.f, v[V];
#pragma unroll
        for (int x = 0; x < 4; ++x) top = fmaxf(top, share[x * 16 * MROW + HD]);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float *m = share + x * 16 * MROW;
            const float k = m[HD] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[HD] - top);
            sum = fmaf(m[HD + 1], k, sum);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = fmaf(m[d0 + e], k, v[e]);
        }
        if (p < this_pairs) {
            if (whole) {
                battn_few_out<V, HD, NP>(a, this_r0, this_kvh, this_pair + p, d0, v, sum);
            } else {
                float *to = slots + (size_t)(2 * w + begins) * battn_few_slot<HD>(PAIRS) + p * MROW;
                store_values<V>(to + d0, v);
                if (d0 == 0) { to[HD] = top; to[HD + 1] = sum; }
            }
        }
        if (!whole && begins && tid == 0)                     // it goes on in the runs behind this one
            merges[w] = FewMerge{battn_run_of(group_end, q, rem) - w + 1, this_r0, this_kvh, this_pair, this_pairs};
        if (!goes_on) return;
        __syncthreads();                                      // (the shares have been read)
    }
}

}  // namespace ks
