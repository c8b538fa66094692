"""Which kernel a batch of trees over a bf16 cache goes to (batch_route.h): that the cases meant for the tiles get there, and tiles side by side where they are meant to be (tile_deal.h)."""
import os
import subprocess

import pytest

from tree_tile_cases import cases

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_16162_amd", "csrc")
PAD = 3                 # rows of the arrays behind the last request's

DRIVER = r'''
#include <cstdio>
#include <cstdlib>
#include "batch_route.h"
#include "tile_deal.h"
int main(int n, char **v) {
    int i = 1;
    auto next = [&] { return atoll(v[i++]); };
    while (i < n) {
        const long long table = next();
        const int dim = (int)next(), group = (int)next(), kv_heads = (int)next(), most_rows = (int)next(), pad = (int)next(), positions = (int)next(), requests = (int)next();
        long long one = 0, all = 0, rows = pad;
        int widest = 0;
        for (int r = 0; r < requests; ++r) {
            const int mine = (int)next(), len = (int)next();
            const ks::TileShape f = ks::tile_shape(mine, len, group, positions, true);
            const int tiles = ks::battn_tiles(f.pairs);
            rows += mine;
            one += f.total();
            all += f.total() * tiles;
            widest = tiles > widest ? tiles : widest;
        }
        const long long most = (most_rows > 0 && most_rows < rows ? most_rows : rows) * group;
        printf("%d %d\n", ks::goes_to_few(true, table, dim, rows, group, requests, kv_heads, most), ks::tiles_side_by_side(widest, one, all));
    }
}
'''


@pytest.fixture(scope="module")
def route(tmp_path_factory):
    tmp = tmp_path_factory.mktemp("route")
    (tmp / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-I", CSRC, "-o", str(tmp / "driver"), str(tmp / "driver.cpp")], check=True)

    def run(c, table, positions):
        args = [table, c["dim"], c["heads"] // c["kv_heads"], c["kv_heads"], max(c["rows"]) if c.get("most") else 0, PAD, positions, len(c["rows"])] + [x for p in zip(c["rows"], c["lens"]) for x in p]
        out = subprocess.run([str(tmp / "driver")] + [str(x) for x in args], check=True, capture_output=True, text=True).stdout.split()
        return out[0] == "1", out[1] == "1"
    return run


def test_the_cases_for_the_tiles_go_there(route):
    for c in cases():
        for positions in (64, 4096 // c["dim"]):              # of a block, bf16 and fp32 caches
            few, side = route(c, c["table"], positions)
            assert not few, c["name"]
            assert c["side"] in (None, side), (c["name"], c["rows"])


def test_few_trees_over_short_contexts_do_not(route):
    c = dict(rows=[26], lens=[1500], heads=40, kv_heads=8, dim=128)
    assert route(c, 1536, 64)[0] and route(c, 4032, 64)[0] and not route(c, 6016, 64)[0]
    assert route(dict(c, rows=[3], most=True), 1 << 30, 64)[0]
