// Attention of a batch's rows on the matrix cores: over pages (PAGED) or over their own prompts' rows.
#pragma once
#include <cfloat>
#include <climits>

#include "battn_common.h"
#include "tile_deal.h"

namespace ks {

// ------------------------------------------------------------------------------------------
// Many rows: tiles of 128 (row, head) pairs of one kv head, 32 per wavefront, on the matrix cores.
// Everything is computed transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane keeps one pair from the scores to the output: the
// accumulators of S^T (position 8(i/4) + 4(lane/32) + i%4 of pair lane%32 in register i) are, rounded and packed as they lie, the operand of the
// second product, whose other operand takes the values' positions in the same order by transposing reads of LDS. Nothing is
// exchanged between lanes but one maximum per block.
// Keys and values come in blocks of 32 or 64 positions straight to LDS, one block ahead.
// What bounds it: over prompts and chunks the vector unit (exponentials, packing) beside the matrix cores, which do not wait for one another within a wavefront but do
// between two products of one; further wavefronts on a SIMD fill that partly (two in all over pages, three over prompts in heads of 128, four in heads of 64). Two prompts of 4096 rows, 40 heads of 128, bf16: 365 us = 941 TFLOP/s (matrix cores busy
// 51 % of the time, the vector unit as much; on zeros, where the power limit leaves more clock, a quarter faster); eight chunks of up to 900 rows over 700 to 9000 positions in pages, 40 heads over 8: 485 us = 783 TFLOP/s. In fp32 the matrix instructions
// themselves: a sixteenth of the bf16 rate.
// ------------------------------------------------------------------------------------------
// What a lane's weights of a block may add up to before their reference follows the scores. Sums of values times weights have that much less room: 2^33 times the blocks of an
// axis, times the values, has to stay below 2^128. Following costs nothing where scores have a standard deviation of 1 or 4; of 8, prompts of 4096 rows take 366 us, as
// with 2^64, with 2^24 374, with 2^16 391 (chunks 475, 489, 532).
constexpr float BT_RISE = 0x1p32f;
// positions of a block: 64, or 32 over prompts in heads of 128, where the registers of a block's scores then leave room for a third wavefront on each SIMD
// (two prompts of 4096 rows 418 -> 400 us; over pages, whose wavefronts need more of them, 512 -> 522 us)
template <int HD, bool PAGED, int NP> constexpr int battn_tile_positions() { return NP == 0 ? 32 * 128 / HD : HD == 128 && !PAGED ? 32 : 64; }

// Tile `index` of the batch: its request and its number in there; false behind the last. Every wavefront for itself, 64 requests at a time.
__device__ __forceinline__ bool battn_find_tile(const BattnArgs &a, int index, int &r_out, int &tile_out, int &tiles_out) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int r0 = 0; r0 < a.n_requests; r0 += 64) {
        const int r = r0 + lane;
        int mine = 0;
        if (r < a.n_requests) mine = (int)(((long long)rows_of(a.row_start, r, a.n_rows).n * a.group + BT_PAIRS - 1) / BT_PAIRS);
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

template <int HD, bool PAGED, int NP> constexpr int battn_tile_lds() { return 2 * 2 * battn_tile_positions<HD, PAGED, NP>() * HD * (NP == 0 ? 4 : 2); }

__device__ __forceinline__ TileShape battn_tile_shape(const BattnArgs &a, int r, int positions, bool side_by_side) {
    const int n = rows_of(a.row_start, r, a.n_rows).n;
    return tile_shape(n, n > 0 ? battn_len(a, r) : 0, a.group, positions, side_by_side);
}

// NP: 1 all in bf16; 3 fp32 queries over a bf16 cache, which stay exact as three bf16 planes, as do the weights; 0 all in fp32, on the fp32 matrix
// instructions (two positions, or dimensions, each), which take keys, values and weights as they lie.
// TREE (pages): of the new rows a row sees those that its mask has, looked at in the last blocks only, the mask's first word in registers. 24 trees of 8 to 64 rows at 200 to 4000
// positions, 40 heads of 128 over 8, bf16: 86 us, 430 TFLOP/s; two of 60 to 64 rows at 100 000 positions: 350 us, 716 TFLOP/s. What bounds them is a block's own chain (arrival, products,
// exponentials, products): a tile takes as long for 2 pairs as for 128.
template <int HD, bool PAGED, int NP, bool TREE>
__global__ __launch_bounds__(256, HD == 128 && !PAGED && NP == 1 ? 3 : 2) void battn_tile_kernel(BattnArgs a) {
    static_assert(PAGED || !TREE, "");
    constexpr int KS = HD / 16, DT = HD / 32, ELT = NP == 0 ? 4 : 2, RB = HD * ELT, SL = RB / 16, MROW = HD + BF_PAD;
    constexpr int CH = battn_tile_positions<HD, PAGED, NP>(), KV = CH * RB;                             // bytes of a block's keys (or values)
    constexpr int ROWS = 64 / SL, NI = KV / 1024 / 4;         // rows a wavefront's load covers, loads per wavefront for the keys
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const unsigned int l0 = (unsigned int)(uintptr_t)BATTN_LDS(lds);
    const float c2 = fmaxf(fabsf(a.scale2), FLT_MIN);         // (a hidden score, -inf, has to stay that under a scale of 0)
    const unsigned int flip = a.scale2 < 0.f ? 0x80000000u : 0u;

    int r = 0, kvh, tile;
    TileShape f{0, 0, 0, false, 0, 0, 0};
    // the run: where it is and where it ends, in cost; the cost before the tile
    long long at = 0, end = 0, before = 0, run_q = 0, run_rem = 0;
    int run = 0;                                              // (its place among the runs that may hold parts of the same tiles)
    int slot_run = 0;                                         // its place in the workspace
    const long long block_cost = (long long)CH * a.group;
    bool side_by_side = false;                                // trees: a kv head's tiles are worked on at once
    int mine_of = 0, most_runs = (int)gridDim.x;              // this workgroup's tile then; runs at most
    if constexpr (PAGED) {
        run = slot_run = battn_run();
        if constexpr (TREE) {
            long long one = 0, all = 0;                       // what a run's workgroups have to do if they are as many as the widest request's tiles, and what of it is work
            int widest = 0;
            for (int q0 = 0; q0 < a.n_requests; q0 += 64) {
                long long cost = 0;
                int tiles = 0;
                if (q0 + lane < a.n_requests) {
                    const TileShape g = battn_tile_shape(a, q0 + lane, CH, true);
                    cost = g.total();
                    tiles = battn_tiles(g.pairs);
                }
                long long tiled = cost * tiles;
                for (int off = 32; off; off >>= 1) {
                    cost += __shfl_xor(cost, off);
                    tiled += __shfl_xor(tiled, off);
                    tiles = max(tiles, __shfl_xor(tiles, off));
                }
                one += cost;
                all += tiled;
                widest = max(widest, tiles);
            }
            one = battn_same(one);
            all = battn_same(all);
            widest = battn_same(widest);
            side_by_side = tiles_side_by_side(widest, one, all);
            if (side_by_side) {
                const TilePlace place = tile_place((int)blockIdx.x, (int)gridDim.x, widest);
                run = place.run;
                slot_run = place.slot_run;
                most_runs = place.most_runs;
                mine_of = place.mine_of;
            }
        }
        if (tid == 0) ((FewMerge *)a.ws)[slot_run] = FewMerge{0, 0, 0, 0, 0};
        long long total = 0;
        for (int pass = 0; pass < 2; ++pass) {
            bool found = false;
            for (int q0 = 0; q0 < a.n_requests && !found; q0 += 64) {
                long long upto = 0;
                if (q0 + lane < a.n_requests) upto = battn_tile_shape(a, q0 + lane, CH, side_by_side).total() * a.Hkv;
                for (int off = 1; off < 64; off <<= 1) {
                    const long long u = __shfl_up(upto, off);
                    if (lane >= off) upto += u;
                }
                if (pass == 0) total += battn_lane(upto, 63);
                if (pass == 0 && q0 + 64 >= a.n_requests) {   // the total is known
                    if (total == 0) return;
                    const int runs = battn_same((int)max(1ll, min((long long)most_runs, battn_divide(total, block_cost))));
                    if (run >= runs) return;
                    run_q = battn_divide(total, runs);
                    run_rem = total - run_q * runs;
                    at = battn_same(run * run_q + min((long long)run, run_rem));
                    end = battn_same((run + 1) * run_q + min((long long)run + 1, run_rem));
                }
                if (pass == 1 || a.n_requests <= 64) {
                    const unsigned long long past = __ballot(at < before + upto);
                    found = past != 0;
                    if (found) {
                        const int src = __builtin_ctzll(past);
                        r = q0 + src;
                        if (src > 0) before += battn_lane(upto, src - 1);
                    } else {
                        before += battn_lane(upto, 63);
                    }
                }
            }
            if (found) break;
        }
        f = battn_tile_shape(a, r, CH, side_by_side);
        kvh = (int)battn_divide(at - before, f.total());
        before += kvh * f.total();
        int lo = 0, hi = f.tiles;
        while (hi - lo > 1) {                                 // the last tile that begins at or before `at`
            const int mid = (lo + hi) >> 1;
            if (before + f.before(mid) <= at) lo = mid;
            else hi = mid;
        }
        tile = lo;
        before += f.before(tile);
    } else {
        kvh = blockIdx.x % a.Hkv;                             // (a kv head's tiles run behind few L2s)
        if (!battn_find_tile(a, blockIdx.x / a.Hkv, r, tile, f.tiles)) return;
        tile = f.tiles - 1 - tile;                            // a request's long ones first (the requests in their own order)
        f.n = rows_of(a.row_start, r, a.n_rows).n;
        f.pairs = (long long)f.n * a.group;
    }
    int buf = 0;                                              // where the next block goes
    // the segment: blocks [b0, b1) of a tile
    int r0, n, len, last, base, b0, b1, n_blocks;
    const char *kb, *vb;
    const_ints table;
    // first row of the wavefront's i-th load of block c (rows past the request's last repeat that one)
    auto load_row = [&](int c, int i) __attribute__((always_inline)) { return min(c * CH + (i * 4 + wave) * ROWS, last & -ROWS); };
    // order of a row's 16-byte pieces (exclusive or with these), so that LDS reads do not meet in one of its 64 banks: the keys' are 32 rows, two pieces of each,
    // the values' four rows, four pieces of each, or (fp32) two rows four apart, eight pieces of each, at a time
    auto key_order = [](int row) { return RB >= 256 ? row & 15 : (row >> 1) & 7; };
    auto value_order = [](int row) { return NP == 0 ? (row & 4) << 1 : HD == 128 ? (row & 3) << 2 : (row & 2) << 1; };
    const int kpiece = (lane % SL) ^ key_order(wave * ROWS + lane / SL), vpiece = (lane % SL) ^ value_order(wave * ROWS + lane / SL);
    int page[NI];
    auto look_up = [&](int c) __attribute__((always_inline)) {                               // the pages of block c
        if constexpr (PAGED)
#pragma unroll
            for (int i = 0; i < NI; ++i) page[i] = table[load_row(c, i) >> a.shift];
    };
    auto issue = [&](int c, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int b = load_row(c, i), in = min(lane / SL, last - b);
            const unsigned int d = l0 + buf * 2 * KV + (i * 4 + wave) * 1024;
            const int kp = 16 * (kpiece ^ (key_order(i * 4 * ROWS) & 8));     // (eight rows a load of all wavefronts: every other one has the order's top bit)
            if constexpr (PAGED) {
                const int pg = (unsigned)page[i] < (unsigned)a.n_pages ? page[i] : 0;
                const long long at = (pg * a.page_stride + (b & ((1 << a.shift) - 1)) * a.pos_stride) * ELT;
                const unsigned int off = (unsigned int)in * (unsigned int)a.pos_stride * ELT;
                battn_dma(kb + at, off + kp, d);
                battn_dma(vb + at, off + vpiece * 16, d + KV);
            } else {
                battn_dma(kb + b * a.k_stride * ELT, (unsigned int)in * (unsigned int)a.k_stride * ELT + kp, d);
                battn_dma(vb + b * a.v_stride * ELT, (unsigned int)in * (unsigned int)a.v_stride * ELT + vpiece * 16, d + KV);
            }
        }
    };
    // where the lane reads in a block: keys of position col, dimensions 16 ks + 8 half ...; values of position 4 half + (lane % 16) / 4 (and 8 on), four
    // dimensions from 32 dt + 16 (lane / 16 % 2) + 4 (lane % 4). fp32: dimensions 8 ks + 4 half ...; position 4 half, dimension 32 dt + col
    constexpr int KR = NP == 0 ? HD / 8 : KS;                 // the lane's reads of a position's keys
    unsigned int k_at[KR], v_at[DT];
#pragma unroll
    for (int ks = 0; ks < KR; ++ks) k_at[ks] = l0 + col * RB + (((2 * ks + half) ^ key_order(col)) * 16);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        const int v_row = 4 * half + (NP == 0 ? 0 : (lane & 15) >> 2), v_col = NP == 0 ? col : 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
        v_at[dt] = l0 + KV + v_row * RB + (((32 * dt + v_col) * ELT / 16) ^ value_order(v_row)) * 16 + v_col * ELT % 16;
    }
    auto enter = [&]() __attribute__((always_inline)) {       // the segment of `tile` that begins at `at`
        r0 = rows_of(a.row_start, r, a.n_rows).first;
        n = battn_same(f.n);
        len = PAGED ? battn_same(battn_len(a, r)) : n;
        last = len - 1;
        base = len - n;                                       // position of the request's first new row
        const int tile_last = battn_same((int)((f.upto(tile) - 1) / a.group));
        n_blocks = (max(base, 0) + tile_last) / CH + 1;
        b0 = 0;
        b1 = n_blocks;
        kb = (const char *)a.k;
        vb = (const char *)a.v;
        if constexpr (PAGED) {
            const long long cost = f.cost(tile);
            b0 = (int)battn_divide(at - before, block_cost);
            if (end < before + cost) b1 = (int)min((long long)n_blocks, battn_divide(end - before, block_cost));
            b1 = battn_same(b1);
            kb += kvh * a.head_stride * ELT;
            vb += kvh * a.head_stride * ELT;
            table = a.table + (size_t)r * a.width;
        } else {
            kb += ((long long)r0 * a.k_stride + kvh * HD) * ELT;
            vb += ((long long)r0 * a.v_stride + kvh * HD) * ELT;
        }
        if (len > 0 && b0 < b1) {
            look_up(b0);
            issue(b0, buf);
            look_up(b0 + 1);
        }
    };
    // on to the next tile; false behind the run's last
    auto advance = [&]() __attribute__((always_inline)) {
        return tile_advance(f, r, kvh, tile, before, at, end, a.Hkv, a.n_requests, mine_of,
                            [&](int q) __attribute__((always_inline)) { return battn_tile_shape(a, q, CH, side_by_side); },
                            [](long long v) __attribute__((always_inline)) { return battn_same(v); });
    };
    if constexpr (TREE)
        if (side_by_side && mine_of >= battn_tiles(f.pairs) && !advance()) return;         // the request has no such tile
    enter();
    while (b0 < b1) {
        const long long p0 = (long long)(side_by_side ? mine_of : tile) * BT_PAIRS;
        const int wave_first = battn_same((int)((p0 + wave * 32) / a.group));                                     // the wavefront's first row
        const int wave_last = battn_same(p0 + wave * 32 < f.pairs ? (int)((min(p0 + wave * 32 + 32, f.pairs) - 1) / a.group) : INT_MIN / 2);      // ... and last one
        const long long pair = min(p0 + wave * 32 + col, f.pairs - 1);
        const bool live = p0 + wave * 32 + col < f.pairs;
        const int row = (int)(pair / a.group), g = (int)(pair - (long long)row * a.group);
        const int limit = base + row;                         // the lane's last visible position
        bf16x8_t qf[KS][NP == 0 ? 1 : NP];                    // dimensions 16 ks + 8 half ... of the lane's pair
        f32x4_t qs[NP == 0 ? KR : 1];                         // fp32: 8 ks + 4 half ...
        {
            const long long q_at = (long long)(r0 + row) * a.q_stride + (kvh * a.group + g) * HD + half * (NP == 0 ? 4 : 8);
            if constexpr (NP == 0) {
#pragma unroll
                for (int ks = 0; ks < KR; ++ks) qs[ks] = __builtin_bit_cast(f32x4_t, *reinterpret_cast<const u32x4_t *>((const float *)a.q + q_at + ks * 8) ^ flip);
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    if constexpr (NP == 1) {
                        qf[ks][0] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t *>((const bf16_t *)a.q + q_at + ks * 16) ^ (flip | flip >> 16));
                    } else {
                        const u32x4_t lo = *reinterpret_cast<const u32x4_t *>((const float *)a.q + q_at + ks * 16) ^ flip, hi = *reinterpret_cast<const u32x4_t *>((const float *)a.q + q_at + ks * 16 + 4) ^ flip;
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 4; ++e) { v[e] = __uint_as_float(lo[e]); v[4 + e] = __uint_as_float(hi[e]); }
                        battn_planes<3>(v, qf[ks]);
                    }
                }
            }
        }
        BattnMask mask{};
        if constexpr (TREE) mask = battn_mask(a, r0 + row);
        float ref = -INFINITY, l = 0.f;
        f32x16_t o[DT];
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
        // block c is here, nobody reads block c-1 any more, and the next one is on its way
        auto arrive = [&](int c) __attribute__((always_inline)) {
            battn_wait<0>();
            battn_meet();
            if (c + 1 < b1) {
                issue(c + 1, buf ^ 1);
                look_up(c + 2);
            }
        };
        auto scores = [&](int c, f32x16_t *s) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < CH / 32; ++t) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KR; ++ks) {
                    unsigned int from = k_at[ks] + buf * 2 * KV;
                    asm("" : "+v"(from));                     // (one address, the tiles by the read's own offset)
                    const u32x4_t kf = *(__attribute__((address_space(3))) const u32x4_t *)(uintptr_t)(from + t * 32 * RB);
                    if constexpr (NP == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kf[e]), qs[ks][e], s[t], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int q = NP - 1; q >= 0; --q) s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[ks][q], s[t], 0, 0, 0);
                    }
                }
            }
            if constexpr (TREE) {
                if (c * CH + CH > base) {               // the block has new rows
                    const unsigned long long seen = mask.seen(c * CH - base, row) >> (4 * half);
#pragma unroll
                    for (int t = 0; t < CH / 32; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!(seen >> (t * 32 + 8 * (i / 4) + i % 4) & 1)) s[t][i] = -INFINITY;
                }
            } else if (c * CH + CH - 1 > base + wave_first) {  // some of the block's positions lie behind some of the wavefront's rows
#pragma unroll
                for (int t = 0; t < CH / 32; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c * CH + t * 32 + 8 * (i / 4) + 4 * half + i % 4 > limit) s[t][i] = -INFINITY;
            }
        };
        // the reference becomes the largest score
        auto follow = [&](const f32x16_t *s) __attribute__((always_inline)) {
            float cm = s[0][0];
#pragma unroll
            for (int t = 0; t < CH / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) cm = fmaxf(cm, s[t][i]);
            cm = fmaxf(cm, lane_xor(cm, 32));
            const float now = fmaxf(ref, battn_rounded_product(cm, c2)), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            l *= f;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[t] *= f;
        };
        auto weigh = [&](f32x16_t *s) __attribute__((always_inline)) {
            const float off = ref == -INFINITY ? 0.f : ref;
            float ps = 0.f;
#pragma unroll
            for (int t = 0; t < CH / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[t][i] = __builtin_amdgcn_exp2f(fmaf(s[t][i], c2, -off));
                    ps += s[t][i];
                }
            return ps;
        };
        // The weights are taken against the largest score of the tile's first block: what comes later may be above that, its weights more than 1 (bf16 and
        // fp32 have the same steps there), before the reference has to follow. So a block's weights wait for no maximum; a block whose sum shows that it should
        // have been looked for is begun anew, and so is one behind blocks whose scores were all -inf, however low its own are.
        auto work = [&](int c, auto first_) __attribute__((always_inline)) {
            constexpr bool FIRST = decltype(first_)::value;
            f32x16_t s[CH / 32];
            scores(c, s);
            if constexpr (FIRST) follow(s);
            float ps = weigh(s);
            if (!FIRST && __builtin_expect(__any(ps > BT_RISE || ref == -INFINITY), 0)) {
                scores(c, s);
                follow(s);
                ps = weigh(s);
            }
            l += ps;
            unsigned int from[DT];
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                from[dt] = v_at[dt] + buf * 2 * KV;
                asm("" : "+v"(from[dt]));
            }
            if constexpr (NP == 0) {
#pragma unroll
                for (int t = 0; t < CH / 32; ++t)
#pragma unroll
                    for (int i = 0; i < 16; ++i)              // position 8 (i/4) + i%4 and four on: a weight is an operand as it lies
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            const float vf = *(__attribute__((address_space(3))) const float *)(uintptr_t)(from[dt] + (t * 32 + 8 * (i / 4) + i % 4) * RB);
                            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, s[t][i], o[dt], 0, 0, 0);
                        }
            } else {
#pragma unroll
                for (int st = 0; st < CH / 16; ++st) {                  // 16 positions
                    const int t = st >> 1, i0 = (st & 1) * 8;
                    const float pv[8] = {s[t][i0], s[t][i0 + 1], s[t][i0 + 2], s[t][i0 + 3], s[t][i0 + 4], s[t][i0 + 5], s[t][i0 + 6], s[t][i0 + 7]};
                    bf16x8_t pb[NP == 0 ? 1 : NP];
                    battn_planes<NP>(pv, pb);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(uintptr_t)(from[dt] + st * 16 * RB));
                        const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)(uintptr_t)(from[dt] + st * 16 * RB + 8 * RB));
                        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                        for (int q = NP - 1; q >= 0; --q) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[q], o[dt], 0, 0, 0);
                    }
                }
            }
        };
        const int stop = len > 0 ? b1 : b0;                   // (a request without positions: nothing to see)
        const int mine = max(b0, min(stop, (base + wave_last) / CH + (base + wave_last >= 0)));       // blocks from here on lie behind all of the wavefront's rows
        if (b0 < mine) {
            arrive(b0);
            work(b0, std::true_type{});
            buf ^= 1;
            for (int c = b0 + 1; c < mine; ++c, buf ^= 1) {
                arrive(c);
                work(c, std::false_type{});
            }
        }
        for (int c = mine; c < stop; ++c, buf ^= 1) arrive(c);
        l += lane_xor(l, 32);
        const bool whole = b0 == 0 && b1 == n_blocks;
        const int out_row = r0 + row, out_kvh = kvh;
        bool goes_on = false;
        if constexpr (PAGED) {
            if (!whole && b0 == 0 && tid == 0)                // it goes on in the runs behind this one
                ((FewMerge *)a.ws)[slot_run] = FewMerge{battn_run_of(before + f.cost(tile) - 1, run_q, run_rem) - run + 1, r0, kvh,
                                                        (int)p0, (int)min((long long)BT_PAIRS, f.pairs - p0)};
        }
        const int slot = 2 * slot_run + (b0 == 0);
        // on to the next tile: its first block is on its way while this one is written (the buffer that it goes to has been read by all)
        if constexpr (PAGED) {
            goes_on = advance();
            if (goes_on) enter();
        }
        if (!live) {
        } else if (!PAGED || whole) {
            const float inv = l > 0.f ? 1.f / l : 0.f;
            const long long out_at = (long long)out_row * a.out_stride + (out_kvh * a.group + g) * HD + 4 * half;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const float v[4] = {o[t][4 * b] * inv, o[t][4 * b + 1] * inv, o[t][4 * b + 2] * inv, o[t][4 * b + 3] * inv};
                    if constexpr (NP == 1) store_values<4>((bf16_t *)a.out + out_at + t * 32 + b * 8, v);
                    else store_values<4>((float *)a.out + out_at + t * 32 + b * 8, v);
                }
        } else {
            float *to = (float *)((char *)a.ws + battn_few_merges()) + (size_t)slot * battn_few_slot<HD>(BT_PAIRS) + (wave * 32 + col) * MROW;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    *reinterpret_cast<f32x4_t *>(to + t * 32 + b * 8 + 4 * half) = f32x4_t{o[t][4 * b], o[t][4 * b + 1], o[t][4 * b + 2], o[t][4 * b + 3]};
            if (half == 0) { to[HD] = ref; to[HD + 1] = l; }
        }
        if (!goes_on) return;
    }
}

}  // namespace ks
