"""knnssd_tree_plan and knnssd_tree_attention against plain forms in 64 bits."""
import random

import pytest
import torch

import batch_common as B
import tree_common as T
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("rows,words,shape", [([1], 1, "tree"), ([26], 1, "tree"), ([5, 0, 64, 1, 63], 1, "forest"), ([64], 1, "chain"), ([65, 3, 128, 0, 127], 2, "tree"),
                                              ([200, 1, 320], 5, "chain"), ([1024, 7, 1000], 16, "tree"), ([1024], 16, "chain"), ([700], 16, "forest"), ([300], 16, "star"),
                                              ([70, 3], 1, "tree"), ([1500, 20], 16, "tree"), ([130], 2, "chain")])
def test_plan(rows, words, shape):
    rng = random.Random(sum(rows) + words)
    parents = [T.make_parents(rng, n, shape) for n in rows]
    lens = [n + rng.randrange(3000) for n in rows]
    start = [0]
    for n in rows:
        start.append(start[-1] + n)
    pad = 3
    positions = torch.full((start[-1] + pad,), -9, dtype=torch.int32, device="cuda")
    masks = torch.full((start[-1] + pad, words), -9, dtype=torch.int64, device="cuda")
    binding.knnssd_tree_plan(ints(sum(parents, []) + [5] * pad), ints(start), ints(lens), positions, masks)
    want_p, want_m = [], []
    for r, n in enumerate(rows):
        depth, seen = T.plan(parents[r], words)
        most = 64 * words
        want_p += [lens[r] - n + d if i < most else -1 for i, d in enumerate(depth)]
        want_m.append(T.bits([s if i < most else set() for i, s in enumerate(seen)], words))
    assert positions.tolist() == want_p + [-9] * pad
    assert torch.equal(masks[:start[-1]].cpu(), torch.cat(want_m)) and (masks[start[-1]:] == -9).all()


def test_parents_that_are_no_earlier_row():
    parents = [0, 5, -7, 1, 2 ** 31 - 1, -2 ** 31, 5, 7, 6]
    positions, masks = ints([0] * 9), torch.zeros(9, 1, dtype=torch.int64, device="cuda")
    binding.knnssd_tree_plan(ints(parents), ints([0, 9]), ints([9]), positions, masks)
    depth, seen = T.plan(parents, 1)
    assert positions.tolist() == depth and torch.equal(masks.cpu(), T.bits(seen, 1))


def test_lengths_and_row_starts_that_are_wrong():
    """Bounded, not right: nothing outside the batch is written."""
    whole = torch.full((40, 1), -9, dtype=torch.int64, device="cuda")
    at = torch.full((40,), -9, dtype=torch.int32, device="cuda")
    for start, kv in (([0, 5, 2 ** 31 - 1], [3, 2]), ([-2 ** 31, 4, 8], [-5, 2 ** 31 - 1]), ([7, 3, 9], [9, 9]), ([100, 200, 300], [9, 9])):
        binding.knnssd_tree_plan(ints([-1] + [0] * 9), ints(start), ints(kv), at[10:20], whole[10:20])
        torch.cuda.synchronize()
        assert (whole[:10] == -9).all() and (whole[20:] == -9).all() and (at[:10] == -9).all() and (at[20:] == -9).all()


def run(rows, lens, heads, kv_heads, dim, page, q, kv, sets, words, order="head", gap=0, most=False, scale=None):
    """One call and its check. sets: per request, which new rows each row's mask has (bits beyond the row itself among them)."""
    c = B.PagedCase(rows, lens, heads, kv_heads, dim, page, q, kv, order=order, gap=gap, seed=sum(lens))
    pad = c.q.shape[0] - sum(rows)
    masks = torch.cat([T.bits(s, words) for s in sets] + [torch.full((pad, words), -1, dtype=torch.int64)]).cuda()
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, heads, q)
    ws.fill_(255)
    scale = dim ** -0.5 if scale is None else scale
    got = binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws, out=c.out, scale=scale, most_rows=max(rows) if most else 0)
    outs, errs = [], []
    for r, n in enumerate(rows):
        sees = torch.zeros(n, lens[r], dtype=torch.bool)
        sees[:, :max(lens[r] - n, 0)] = True
        for i in range(n):
            for j in sets[r][i]:
                if j <= i and j < 64 * words and 0 <= lens[r] - n + j:
                    sees[i, lens[r] - n + j] = True
        o, e = T.attend64(c.q.cpu()[c.start[r]:c.start[r + 1]], c.k[r], c.v[r], scale, sees, BF16 if q == BF16 else None)
        outs.append(o)
        errs.append(e)
    B.check_rows(got, torch.cat(outs), torch.cat(errs), q)


def trees(rows, shape="tree", seed=0):
    rng = random.Random(seed)
    return [T.plan(T.make_parents(rng, n, shape), 1)[1] for n in rows]


TYPES = [(BF16, BF16), (FP32, BF16), (FP32, FP32)]


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 10, 2), (128, 3, 3), (64, 8, 2), (64, 4, 4), (128, 5, 1), (64, 1, 1)])
@pytest.mark.parametrize("rows,lens", [([1], [1]), ([7], [7]), ([26], [226]), ([3, 0, 64, 1], [3, 5, 164, 700]), ([17, 40], [48, 105]), ([63, 2, 9], [63, 66, 200])])
def test_trees(q, kv, dim, heads, kv_heads, rows, lens):
    run(rows, lens, heads, kv_heads, dim, 16, q, kv, trees(rows, seed=sum(lens)), 1, most=sum(rows) % 2 == 0)


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("page,order", [(8, "head"), (8, "position"), (32, "position"), (64, "head"), (256, "position")])
def test_pages_that_end_inside_a_tree(q, kv, page, order):
    rows, lens = [19, 33, 5], [150, 40, 261]
    run(rows, lens, 8, 4, 64, page, q, kv, trees(rows, "forest"), 1, order=order, gap=1)
    run(rows, lens, 4, 2, 128, page, q, kv, trees(rows, "forest"), 1, order=order, gap=2, most=True)


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows,lens,words", [([100], [100], 2), ([130, 1, 65], [131, 64, 400], 3), ([320], [700], 16), ([90], [90], 1), ([70, 3], [200, 90], 2)])
def test_wide_trees(q, kv, dim, rows, lens, words):
    """Masks of several words; words for more rows than there are; rows that the masks have no bit for."""
    run(rows, lens, 4, 2, dim, 32, q, kv, trees(rows, "tree", 3), words)
    run(rows, lens, 2, 2, dim, 32, q, kv, trees(rows, "star", 3), words, most=True)


def test_the_widest_tree():
    run([1024], [1100], 2, 1, 128, 64, BF16, BF16, trees([1024]), 16)
    run([1030], [1030], 1, 1, 64, 64, BF16, BF16, trees([1030], "chain"), 16)


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("dim,heads,kv_heads", [(128, 4, 2), (64, 2, 2)])
def test_masks_that_are_no_trees(q, kv, dim, heads, kv_heads):
    """Any bits: rows that see nothing at all (an output of 0), rows that do not see themselves, bits of later rows (which stay hidden)."""
    rng = random.Random(5)
    for rows, lens in (([40, 9], [40, 9]), ([12], [12]), ([64, 30], [90, 31]), ([150], [150])):
        sets = [[set() if rng.random() < 0.3 else {j for j in range(n) if rng.random() < 0.2} for _ in range(n)] for n in rows]
        run(rows, lens, heads, kv_heads, dim, 16, q, kv, sets, 3)
    run([20, 3], [20, 3], heads, kv_heads, dim, 16, q, kv, [[set()] * 20, [set()] * 3], 1)


@pytest.mark.parametrize("q,kv", TYPES)
def test_far_positions(q, kv):
    rows, lens = [21, 4], [5000, 9003]
    run(rows, lens, 8, 1, 128, 64, q, kv, trees(rows), 1)
    run(rows, lens, 4, 4, 64, 128, q, kv, trees(rows), 1, order="position")


@pytest.mark.parametrize("q,kv", TYPES)
def test_scales(q, kv):
    for scale in (0.0, -0.2, 1.5):
        run([9, 30], [60, 31], 4, 2, 64, 16, q, kv, trees([9, 30]), 1, scale=scale)


@pytest.mark.parametrize("q,kv", TYPES)
def test_a_length_that_is_less_than_the_rows(q, kv):
    """kv_len below the number of rows: row i is position kv_len - rows + i, those before 0 are none."""
    run([12], [7], 4, 2, 64, 16, q, kv, trees([12], "chain"), 1)
    run([70, 5], [33, 5], 4, 2, 128, 16, q, kv, trees([70, 5], "chain"), 2)


def test_chains_are_what_the_paged_attention_gives():
    """Not bit for bit, and nothing says so: the two are compiled apart, and where products and sums are joined is the compiler's. Each is off the exact result by at most the error that
    fp32 allows (err) and a rounding of half a step of what it then is (|want| + err), so one from the other by at most twice that."""
    for rows, lens, heads, kv_heads, dim, q, kv in (([5, 1, 9], [300, 200, 1000], 10, 2, 128, BF16, BF16), ([40, 64], [300, 64], 8, 8, 64, FP32, BF16), ([7, 30], [90, 400], 4, 2, 64, FP32, FP32)):
        c = B.PagedCase(rows, lens, heads, kv_heads, dim, 16, q, kv)
        pages = binding.Pages(c.k_pages, c.v_pages)
        ws = binding.paged_attention_workspace(pages, heads, q)
        masks = torch.cat([T.bits([set(range(i + 1)) for i in range(n)], 1) for n in rows] + [torch.zeros(3, 1, dtype=torch.int64)]).cuda()
        want = binding.knnssd_paged_attention(pages, c.block_table, c.row_start, c.kv_len, c.q, ws, out=torch.zeros_like(c.q))
        got = binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws, out=torch.zeros_like(c.q))
        outs, errs = zip(*[B.attend64(c.q.cpu()[a:b], c.k[r], c.v[r], dim ** -0.5, BF16 if q == BF16 else None) for r, (a, b) in enumerate(zip(c.start, c.start[1:]))])
        exact, err = torch.cat(outs), torch.cat(errs)
        off = (got.cpu().double() - want.cpu().double())[:sum(rows)].abs()
        assert (off <= 2 * (err + B.half_step(q) * (exact.abs() + err))).all() and torch.equal(got[sum(rows):], want[sum(rows):])


def test_bad_tables_and_lengths_stay_inside():
    """Page ids and lengths that are none: no access out of range (values are whatever they are), and nothing but the rows is written."""
    c = B.PagedCase([5, 30], [40, 90], 4, 2, 64, 16, BF16, BF16, pad=4)
    k, v = torch.nan_to_num(c.k_pages), torch.nan_to_num(c.v_pages)
    pages = binding.Pages(k, v)
    ws = binding.paged_attention_workspace(pages, 4, BF16)
    masks = torch.full((c.q.shape[0], 1), -1, dtype=torch.int64, device="cuda")
    for table, kv_len, start in ((c.block_table * 0 + 2 ** 30, c.kv_len, c.row_start), (c.block_table, ints([2 ** 31 - 1, -4]), c.row_start),
                                 (c.block_table, c.kv_len, ints([-5, 2 ** 31 - 1, 3])), (c.block_table, c.kv_len, ints([30, 10, 35]))):
        out = torch.full_like(c.q, 5.0)
        binding.knnssd_tree_attention(pages, table, start, kv_len, masks, c.q, ws, out=out)
        torch.cuda.synchronize()
    out = torch.full_like(c.q, 5.0)
    binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws, out=out)
    assert (out[35:] == 5.0).all()


def test_refusals():
    c = B.PagedCase([5], [40], 4, 2, 64, 16, BF16, BF16)
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, 4, BF16)
    n = c.q.shape[0]
    good = torch.zeros(n, 1, dtype=torch.int64, device="cuda")
    for masks in (good.int(), good[:n - 1], good[:, 0], good.cpu(), torch.zeros(n, 4, dtype=torch.int64, device="cuda")[:, ::2]):
        with pytest.raises(ValueError, match="masks"):
            binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws)
        with pytest.raises(ValueError, match="masks"):
            binding.knnssd_tree_plan(ints([0] * n), c.row_start, c.kv_len, ints([0] * n), masks)
    with pytest.raises(binding.KnnSsdError):
        binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, torch.zeros(n, 17, dtype=torch.int64, device="cuda"), c.q, ws)
    with pytest.raises(ValueError, match="positions"):
        binding.knnssd_tree_plan(ints([0] * n), c.row_start, c.kv_len, ints([0] * (n - 1)), good)
