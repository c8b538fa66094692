"""Batches of trees for battn_tile_kernel: tables for so many positions that a batch over a bf16 cache goes there (batch_route.h), with what they hold."""
import random

import tree_common as T

FAR = 1 << 20           # positions that a request's table has entries for


def trees(rows, shape="tree", seed=0):
    rng = random.Random(seed)
    return [T.plan(T.make_parents(rng, n, shape), 1)[1] for n in rows]


def any_bits(rows, seed=5):
    """Rows that see nothing at all, rows that do not see themselves, bits of later rows (which stay hidden)."""
    rng = random.Random(seed)
    return [[set() if rng.random() < 0.3 else {j for j in range(n) if rng.random() < 0.2} for _ in range(n)] for n in rows]


def case(name, rows, lens, heads, kv_heads, dim, page=16, sets=None, words=1, side=None, **kw):
    """side: whether a kv head's tiles are worked on side by side (None: either)."""
    return dict(name=name, side=side, rows=rows, lens=lens, heads=heads, kv_heads=kv_heads, dim=dim, page=page, sets=trees(rows, seed=sum(lens)) if sets is None else sets, words=words, table=FAR, **kw)


def cases():
    out = []
    for heads, kv_heads, dim in ((10, 2, 128), (3, 3, 128), (5, 1, 128), (8, 2, 64), (4, 4, 64), (2, 1, 64)):
        for rows, lens in (([26], [226]), ([3, 0, 64, 1], [3, 5, 164, 700]), ([17, 40], [48, 105]), ([63, 2, 9], [63, 66, 200])):
            out.append(case("trees", rows, lens, heads, kv_heads, dim, most=sum(rows) % 2 == 0))
    for page, order in ((8, "head"), (8, "position"), (32, "position"), (64, "head"), (256, "position")):
        rows, lens = [19, 33, 5], [150, 40, 261]
        out.append(case("pages", rows, lens, 8, 4, 64, page, trees(rows, "forest"), order=order, gap=1))
        out.append(case("pages", rows, lens, 4, 2, 128, page, trees(rows, "forest"), order=order, gap=2, most=True))
    for dim in (64, 128):
        for rows, lens, words in (([100], [100], 2), ([130, 1, 65], [131, 64, 400], 3), ([320], [700], 16), ([90], [90], 1), ([70, 3], [200, 90], 2)):
            out.append(case("words", rows, lens, 4, 2, dim, 32, trees(rows, "tree", 3), words))
            out.append(case("words", rows, lens, 2, 2, dim, 32, trees(rows, "star", 3), words, most=True))
        for rows, lens in (([40, 9], [40, 9]), ([24], [24]), ([64, 30], [90, 31]), ([150], [150]), ([150, 20], [1150, 90])):
            out.append(case("any bits", rows, lens, 4, 2, dim, 16, any_bits(rows), 3))
        out.append(case("nothing", [20, 3], [20, 3], 4, 2, dim, 16, [[set()] * 20, [set()] * 3]))
        out.append(case("short", [24], [15], 4, 2, dim, 16, trees([24], "chain")))
        out.append(case("short", [70, 5], [33, 5], 4, 2, dim, 16, trees([70, 5], "chain"), 2))
        for scale in (0.0, -0.2, 1.5):
            out.append(case("scales", [9, 30], [60, 31], 4, 2, dim, scale=scale))
        out.append(case("far", [21, 4], [5000, 9003], 8, 1, dim, 128, order="position"))
        # several tiles side by side, requests of fewer among them; of more than eight tiles, or of too few such requests, one behind the other
        out.append(case("side", [128, 1, 0, 2], [900, 130, 7, 140], 8, 1, dim, 16, trees([128, 1, 0, 2], seed=1), 2, side=True))
        out.append(case("side", [1, 2, 64, 60, 3], [60, 70, 1500, 1400, 75], 16, 2, dim, 64, any_bits([1, 2, 64, 60, 3]), 1, side=True, gap=1))
        out.append(case("side", [320, 1], [2000, 300], 3, 1, dim, 32, trees([320, 1], seed=4), 5, side=True))
        out.append(case("behind", [140, 40], [900, 800], 8, 1, dim, 16, trees([140, 40], seed=1), 3, side=False))
        rows = [64 if r % 9 == 5 else 1 + r % 3 for r in range(80)]
        out.append(case("many", rows, [1500 + r if n == 64 else 40 + r for r, n in enumerate(rows)], 8, 1, dim, 64, trees(rows, seed=6), 1, side=True))
        out.append(case("many", rows, [150 + r for r in range(80)], 8, 1, dim, 64, trees(rows, seed=6), 1, side=False))
    out.append(case("widest", [1024], [1100], 2, 1, 128, 64, trees([1024]), 16, side=False))
    out.append(case("widest", [1030], [1030], 1, 1, 64, 64, trees([1030], "chain"), 16, side=False))
    return out
