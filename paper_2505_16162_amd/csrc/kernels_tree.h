// Trees of drafted tokens: positions and masks of ancestors from the rows' parents (tree_plan_kernel), and the kept path's keys and values put side by
// side in the pages (tree_keep_kernel).
#pragma once
#include "../../include/knnssd.h"
#include "device_ops.h"
#include "rows_range.h"

namespace ks {

struct TreePlanArgs {
    const int *parents;
    const_ints row_start, kv_len;
    unsigned long long *masks;
    int *positions;
    int n_rows, words;
};

// A workgroup per request, a thread per row, 64 rows to a wavefront. mask(i) = {i} and mask(parent(i)). Within a wavefront's 64 rows by doubling: each lane takes over what the lane
// that it points to has gathered, and that lane's pointer, so that six exchanges reach any depth. Where a row's ancestors leave the 64, the first one outside has
// the rest: a row's words are put together from at most one row of each 64 before it. Bound by latency, four dependent loads.
__global__ __launch_bounds__(KNNSSD_MAX_TREE) void tree_plan_kernel(TreePlanArgs a) {
    __shared__ unsigned long long own[KNNSSD_MAX_TREE];       // ancestors among a row's 64
    __shared__ int up[KNNSSD_MAX_TREE], steps[KNNSSD_MAX_TREE];          // the first ancestor outside, or -1; how many there are inside
    const int r = blockIdx.x, i = threadIdx.x, lane = i & 63, nt = blockDim.x;
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const int p = i < rows.n ? a.parents[rows.first + i] : -1, parent = p < i ? max(p, -1) : -1;
    int to = parent >= (i & ~63) ? parent & 63 : -1, out = parent < (i & ~63) ? parent : -1, n = to >= 0;
    unsigned long long m = 1ull << lane;
    while (__any(to >= 0)) {
        const int from = to >= 0 ? to : lane;
        const unsigned int lo = __shfl((unsigned int)m, from), hi = __shfl((unsigned int)(m >> 32), from);
        const int there = __shfl(to, from), out_there = __shfl(out, from), n_there = __shfl(n, from);
        if (to >= 0) {
            m |= (unsigned long long)hi << 32 | lo;
            n += n_there;
            out = out_there;
            to = there;
        }
    }
    own[i] = m;
    up[i] = out;
    steps[i] = n;
    __syncthreads();
    if (i < rows.n) {
        unsigned long long *mask = a.masks + (long long)(rows.first + i) * a.words;
        int depth = 0, at = i;
        for (int w = a.words - 1; w >= 0; --w) {
            unsigned long long v = 0;
            if (at >= 0 && at >> 6 == w) {
                v = own[at];
                depth += steps[at];
                at = up[at];
                depth += at >= 0;
            }
            mask[w] = v;
        }
        a.positions[rows.first + i] = (int)max(-1ll, (long long)a.kv_len[r] - rows.n + depth);
    }
    for (int x = i + nt; x < rows.n; x += nt) {               // rows that the masks have no bit for
        for (int w = 0; w < a.words; ++w) a.masks[(long long)(rows.first + x) * a.words + w] = 0;
        a.positions[rows.first + x] = -1;
    }
}

constexpr int KEEP_BLOCKS = 64, KEEP_NT = 256, KEEP_U = 4;    // blocks of a launch, threads, entries under way

typedef unsigned int keep_piece __attribute__((ext_vector_type(4)));
struct TreeKeepArgs {
    void *k[KEEP_BLOCKS], *v[KEEP_BLOCKS];
    long long page_stride, head_stride, pos_stride;           // in bytes
    const_ints table, row_start, kv_len, path, n_path;
    int *cached;                                              // NULL: another launch writes it
    int n_rows, width, shift, n_pages;
    int pieces, head_pieces;                                  // 16-byte pieces of a position's keys, of a head
};

// A workgroup takes a request's path in one block, a thread one 16-byte piece of a position's keys or values all the way along it. The path ascends, so entry j goes to a
// place at or before the one it comes from, and no later entry comes from a place that has been written: a thread needs nobody else's work, and the entries that it
// has under way are read before the first of them is written.
__global__ __launch_bounds__(KEEP_NT) void tree_keep_kernel(TreeKeepArgs a) {
    const int r = blockIdx.x, piece = blockIdx.z * KEEP_NT + threadIdx.x;
    const RowsRange rows = rows_of(a.row_start, r, a.n_rows);
    const long long base = (long long)a.kv_len[r] - rows.n;
    const int count = base < 0 ? 0 : min(a.n_path[r], rows.n);
    const int side = piece >= a.pieces, in = piece - side * a.pieces, head = in / a.head_pieces;
    char *at = (char *)(side ? a.v[blockIdx.y] : a.k[blockIdx.y]) + head * a.head_stride + (in - head * a.head_pieces) * 16;
    const bool mine = piece < 2 * a.pieces;
    const long long held = (long long)a.width << a.shift;
    int kept = 0, last = -1;
    bool more = count > 0;
    for (int j0 = 0; more; j0 += KEEP_U) {
        long long from[KEEP_U], to[KEEP_U];
        bool moves[KEEP_U];
#pragma unroll
        for (int u = 0; u < KEEP_U; ++u) {
            moves[u] = false;
            from[u] = to[u] = 0;
            if (!more) continue;
            const int j = j0 + u, i = j < count ? a.path[rows.first + j] : -1;
            if (i <= last || i >= rows.n || base + i >= held) {
                more = false;                                 // the path's end, or an entry that is none
                continue;
            }
            last = i;
            kept = j + 1;
            if (i == j) continue;
            const long long p = base + i, t = base + j;
            const int pg = a.table[(long long)r * a.width + (p >> a.shift)], tg = a.table[(long long)r * a.width + (t >> a.shift)];
            if ((unsigned)pg >= (unsigned)a.n_pages || (unsigned)tg >= (unsigned)a.n_pages) continue;
            from[u] = pg * a.page_stride + (p & ((1 << a.shift) - 1)) * a.pos_stride;
            to[u] = tg * a.page_stride + (t & ((1 << a.shift) - 1)) * a.pos_stride;
            moves[u] = mine;
        }
        keep_piece x[KEEP_U];
#pragma unroll
        for (int u = 0; u < KEEP_U; ++u)
            if (moves[u]) x[u] = *reinterpret_cast<const keep_piece *>(at + from[u]);
#pragma unroll
        for (int u = 0; u < KEEP_U; ++u)
            if (moves[u]) *reinterpret_cast<keep_piece *>(at + to[u]) = x[u];
    }
    if (a.cached && blockIdx.y == 0 && piece == 0) a.cached[r] = (int)(max(base, 0ll) + kept);
}

}  // namespace ks
