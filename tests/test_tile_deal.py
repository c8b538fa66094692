"""How the tiles of a batch over pages are dealt out (tile_deal.h): every tile's blocks once, no tile that there is not, and no more tiles begun than the merge has places for."""
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_16162_amd", "csrc")

# What battn_tile_kernel does with a run, but for the work: the segments of all workgroups, one line each.
DRIVER = r'''
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "tile_deal.h"
using namespace ks;
int main(int n, char **v) {
    int i = 1;
    while (i + 4 < n) {
        const int group = atoi(v[i]), kv_heads = atoi(v[i + 1]), positions = atoi(v[i + 2]), trees = atoi(v[i + 3]), requests = atoi(v[i + 4]), grid = 512;
        std::vector<int> rows, len;
        for (int r = 0; r < requests; ++r) { rows.push_back(atoi(v[i + 5 + 2 * r])); len.push_back(atoi(v[i + 6 + 2 * r])); }
        i += 5 + 2 * requests;
        long long one = 0, all = 0, total = 0;
        int widest = 0;
        for (int r = 0; r < requests; ++r) {
            const TileShape f = tile_shape(rows[r], len[r], group, positions, true);
            const int tiles = battn_tiles(f.pairs);
            one += f.total();
            all += f.total() * tiles;
            widest = tiles > widest ? tiles : widest;
        }
        const bool side = trees && tiles_side_by_side(widest, one, all);
        auto shape_of = [&](int r) { return tile_shape(rows[r], len[r], group, positions, side); };
        for (int r = 0; r < requests; ++r) total += shape_of(r).total() * kv_heads;
        printf("case %d\n", side);
        for (int w = 0; w < grid; ++w) {
            TilePlace place{(w & 7) * (grid >> 3) + (w >> 3), (w & 7) * (grid >> 3) + (w >> 3), grid, 0};
            if (side) place = tile_place(w, grid, widest);
            printf("place %d\n", place.slot_run);
            long long cost = (long long)positions * group, runs = total / cost < place.most_runs ? total / cost : place.most_runs;
            if (runs < 1) runs = 1;
            if (total == 0 || place.run >= runs) continue;
            const long long q = total / runs, rem = total - q * runs;
            long long at = place.run * q + (place.run < rem ? place.run : rem), end = at + q + (place.run < rem), before = 0;
            int r = 0, kvh = 0, tile = 0;
            TileShape f = shape_of(0);
            while (at >= before + f.total() * kv_heads) { before += f.total() * kv_heads; f = shape_of(++r); }
            kvh = (int)((at - before) / f.total());
            before += kvh * f.total();
            while (tile + 1 < f.tiles && before + f.before(tile + 1) <= at) ++tile;
            before += f.before(tile);
            auto advance = [&] { return tile_advance(f, r, kvh, tile, before, at, end, kv_heads, requests, place.mine_of, shape_of, [](long long x) { return x; }); };
            if (side && place.mine_of >= battn_tiles(f.pairs) && !advance()) continue;
            do {
                const int cached = len[r] > f.n ? len[r] - f.n : 0, blocks = (int)((cached + (f.upto(tile) - 1) / group) / positions + 1);
                const int b0 = (int)((at - before) / cost), b1 = end < before + f.cost(tile) && (end - before) / cost < blocks ? (int)((end - before) / cost) : blocks;
                if (b0 >= b1) break;
                printf("segment %d %d %d %d %d %d %d\n", place.slot_run, r, kvh, side ? place.mine_of : tile, b0, b1, blocks);
            } while (advance());
        }
    }
}
'''


@pytest.fixture(scope="module")
def deal(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("deal")
    (tmp / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", CSRC, "-o", str(tmp / "driver"), str(tmp / "driver.cpp")], check=True)

    def run(group, kv_heads, positions, trees, rows, lens):
        args = [group, kv_heads, positions, trees, len(rows)] + [x for pair in zip(rows, lens) for x in pair]
        out = subprocess.run([str(tmp / "driver")] + [str(x) for x in args], check=True, capture_output=True, text=True).stdout.splitlines()
        return out[0] == "case 1", [int(x.split()[1]) for x in out if x.startswith("place")], [tuple(map(int, x.split()[1:])) for x in out if x.startswith("segment")]
    return run


def check(deal, group, kv_heads, positions, trees, rows, lens):
    side, places, segments = deal(group, kv_heads, positions, trees, rows, lens)
    assert sorted(places) == list(range(512))                 # each workgroup its own
    tiles = {(r, h, t): [] for r, n in enumerate(rows) for h in range(kv_heads) for t in range(-(-n * group // 128))}
    for place, r, h, t, b0, b1, blocks in segments:
        assert (r, h, t) in tiles, "a tile that there is not"
        tiles[r, h, t].append((b0, b1, place, blocks))
    begun = 0
    for at, parts in tiles.items():
        parts.sort()
        assert parts and parts[0][0] == 0 and parts[-1][1] == parts[-1][3], at
        assert all(a[1] == b[0] and a[2] + 1 == b[2] for a, b in zip(parts, parts[1:])), at          # in places one behind the other, as they are joined
        begun += len(parts) > 1
    assert begun <= (-(-sum(rows) * group // 128) + len(rows)) * kv_heads
    return side


def test_tiles_side_by_side_of_requests_that_have_fewer(deal):
    for kv_heads in (1, 2, 8):
        for positions in (32, 64):
            for rows, lens in (([128, 1], [8128, 2001]), ([64, 4, 60, 2], [8064, 2004, 8060, 2000]), ([1, 128, 1, 0, 1], [900, 8128, 700, 5, 1000])):
                assert check(deal, 8, kv_heads, positions, 1, rows, lens)
                assert not check(deal, 8, kv_heads, positions, 0, rows, lens)


@pytest.mark.parametrize("widest", [40, 128, 1024])
def test_batches(deal, widest):
    rng = random.Random(widest)
    side = 0
    for _ in range(200):
        n = rng.randint(1, 6)
        rows = [rng.choice([x for x in (0, 1, 3, 17, 26, 40, 64, 100, 128, 200, 1024) if x <= widest]) for _ in range(n)]
        lens = [max(0, r + rng.choice([-5, 0, 50, 700, 3000, 9000, 30000])) for r in rows]
        side += check(deal, rng.choice([1, 4, 5, 8]), rng.choice([1, 2, 8]), rng.choice([32, 64]), int(rng.random() < 0.8), rows, lens)
    assert side > 20 or widest == 1024


def test_long_contexts(deal):
    """Positions beyond 2^24 count as so many; sums of costs pass 32 bits."""
    for trees in (0, 1):
        check(deal, 8, 8, 64, trees, [64, 60], [100_000, 110_000])
        check(deal, 5, 8, 64, trees, [3, 900], [2 ** 24 + 7, 2 ** 23])
