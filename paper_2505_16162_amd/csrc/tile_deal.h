// How the tiles of a batch over pages are dealt to the workgroups of battn_tile_kernel: plain code, no HIP.
#pragma once

#define KS_DEAL __attribute__((always_inline)) constexpr

namespace ks {

constexpr int BT_PAIRS = 128;
constexpr int BT_FAR = 1 << 24;         // positions beyond count as so many

KS_DEAL int battn_tiles(long long pairs) { return (int)((pairs + BT_PAIRS - 1) / BT_PAIRS); }

// Over pages the batch's tiles are dealt to the workgroups in equal runs, as in battn_few_kernel, by their cost: a tile's is the positions before its request's
// new rows times the heads of a group, and the pairs up to its own last one (a pair's rows counted exactly), or a block's cost, positions of a block times heads
// of a group, if that is more. It is at most what its blocks hold, so a run that begins x into a tile begins with block
// x / (a block's cost) of it, and a run of a block's cost or more is never empty. The costs before a tile have a closed form.
struct TileShape {
    int n, tiles, small;                // rows, tiles of a kv head, those of its first that cost a block
    bool side_by_side;                  // one cost for all of a kv head's tiles (`tiles` is 1): they are worked on at once
    long long step, pairs, block;       // cost of a tile without its own pairs; all pairs; a block's cost
    KS_DEAL long long sloped(int t) const { return t * step + (long long)(BT_PAIRS / 2) * t * (t + 1); }
    KS_DEAL long long before(int t) const { return t <= small ? t * block : small * block + sloped(t) - sloped(small); }      // (t < tiles)
    KS_DEAL long long upto(int t) const { return side_by_side || (t + 1ll) * BT_PAIRS > pairs ? pairs : (t + 1ll) * BT_PAIRS; }      // pairs up to the tile's last
    KS_DEAL long long cost(int t) const { return step + upto(t) > block ? step + upto(t) : block; }
    KS_DEAL long long total() const { return tiles ? before(tiles - 1) + cost(tiles - 1) : 0; }
};
// of a request of n rows and len positions, `positions` to a block
KS_DEAL TileShape tile_shape(int n, int len, int group, int positions, bool side_by_side) {
    TileShape f{0, 0, 0, side_by_side, 0, 0, (long long)positions * group};
    if (n > 0) {
        f.n = n;
        f.pairs = (long long)n * group;
        f.tiles = side_by_side ? 1 : battn_tiles(f.pairs);
        const int cached = len > n ? len - n : 0;
        f.step = (long long)(cached < BT_FAR ? cached : BT_FAR) * group;
        const long long small = f.block > f.step ? (f.block - f.step) / BT_PAIRS : 0;
        f.small = small < f.tiles ? (int)small : f.tiles;
    }
    return f;
}

// Trees: the tiles of a kv head side by side, each in a workgroup of its own over the same positions, so that what one of them reads is in the die's L2 for the others. Then a
// run is a stretch of positions, and as many workgroups of one die share it as the batch's widest request has tiles.
// Only where three quarters of those workgroups have a tile. `one`: what a run's workgroups have to do; `all`: what of it, times their number, is work. Whole calls, us, one tile
// after the other / side by side, 40 heads of 128 over 8, bf16: two requests of 60 to 64 rows at 100 000 positions, three tiles, 381 / 343; three of two tiles 430 / 337; four of 8 to 64 rows at
// 8000 to 40 000 positions (95 % of the workgroups have one) 177 / 171; 24 requests of 8 to 64 rows at 200 to 4000 positions, one to three tiles (65 %), 91 / 120. There wide trees lose a little
// too: 24 of 30 to 64 rows (80 %) 94 / 99, of 40 to 64 (89 %) 133 / 135.
KS_DEAL bool tiles_side_by_side(int widest, long long one, long long all) { return widest > 1 && widest <= 8 && all * 4 >= one * widest * 3; }

// A workgroup's place: its run, the run's place in the workspace, runs at most, and the tile that it takes of each kv head.
struct TilePlace { int run, slot_run, most_runs, mine_of; };
constexpr int BT_NO_RUN = 0x7fffffff;   // (workgroups left over)
KS_DEAL TilePlace tile_place(int block, int grid, int widest) {
    const int slots = grid >> 3, per = slots / widest, die = block & 7, slot = block >> 3, most = 8 * per;
    const int mine_of = slot % widest, run = die * per + slot / widest;
    if (slot >= per * widest) return TilePlace{BT_NO_RUN, most * widest + die * (slots - per * widest) + slot - per * widest, most, mine_of};
    return TilePlace{run, mine_of * most + run, most, mine_of};
}

// On to the next tile of the run that ends at `end`; false behind its last. Side by side, requests that have no tile mine_of are passed over.
template <typename ShapeOf, typename Same>
KS_DEAL bool tile_advance(TileShape &f, int &r, int &kvh, int &tile, long long &before, long long &at, long long end, int kv_heads, int n_requests, int mine_of,
                          const ShapeOf &shape_of, const Same &same) {
    do {
        before = same(before + f.cost(tile));
        if (before >= end) return false;
        at = before;
        if (++tile == f.tiles) {
            tile = 0;
            if (++kvh == kv_heads) {
                kvh = 0;
                do {
                    if (++r >= n_requests) return false;      // (never: the run lies in some requests)
                    f = shape_of(r);
                } while (f.tiles == 0);
            }
        }
    } while (f.side_by_side && mine_of >= battn_tiles(f.pairs));
    return true;
}

}  // namespace ks
