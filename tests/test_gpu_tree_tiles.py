"""knnssd_tree_attention in tiles of 128 pairs (battn_tile_kernel with masks), where tables are so wide that a batch over a bf16 cache goes there: against plain forms in 64 bits."""
import pytest
import torch

import batch_common as B
import tree_common as T
from paper_2505_16162_amd import binding
from test_gpu_tree_attention import BF16, TYPES
from tree_tile_cases import FAR, cases, trees

pytestmark = pytest.mark.gpu
CASES = cases()


def widen(c, table, page):
    """Entries for `table` positions in all, those behind a request's own of ids that are none."""
    extra = max(0, -(-table // page) - c.block_table.shape[1])
    c.block_table = torch.cat([c.block_table, torch.full((len(c.rows), extra), 2 ** 30, dtype=torch.int32, device="cuda")], 1)


def run(rows, lens, heads, kv_heads, dim, page, q, kv, sets, words, order="head", gap=0, most=False, scale=None, table=0, pad=3):
    """One call and its check: every row's output (they all hold 5 before) and the rows behind the last request's. sets: per request, which new rows each row's mask has; table:
    positions that a request's table has entries for (beyond its own: ids that are none)."""
    c = B.PagedCase(rows, lens, heads, kv_heads, dim, page, q, kv, order=order, gap=gap, seed=sum(lens), pad=pad)
    widen(c, table, page)
    masks = torch.cat([T.bits(s, words) for s in sets] + [torch.full((pad, words), -1, dtype=torch.int64)]).cuda()
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, heads, q)
    ws.fill_(255)
    scale = dim ** -0.5 if scale is None else scale
    got = binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws, out=c.out, scale=scale, most_rows=max(rows) if most else 0)
    outs, errs = [], []
    for r, n in enumerate(rows):
        if n == 0:
            continue
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


# requests whose widest has several tiles of a kv head and others that have fewer, most of the work being the widest's, so that a kv head's tiles are worked on side by side
SIDE_BY_SIDE = [([128, 1], [8128, 2001]), ([64, 4, 60, 2], [8064, 2004, 8060, 2000]), ([1, 128, 1, 0, 1], [900, 8128, 700, 0, 1000])]


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("kv_heads", [1, 2])
@pytest.mark.parametrize("rows,lens", SIDE_BY_SIDE)
def test_tiles_side_by_side_of_requests_that_have_fewer(q, kv, kv_heads, rows, lens):
    """A workgroup whose tile the next request does not have goes on behind it. All rows are written, whichever runs their tiles lie in."""
    run(rows, lens, 8 * kv_heads, kv_heads, 128, 64, q, kv, trees(rows, seed=2), 2)


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("name", sorted({c["name"] for c in CASES}))
def test_cases(q, kv, name):
    for c in CASES:
        if c["name"] == name:
            run(**{k: v for k, v in c.items() if k not in ("name", "side")}, q=q, kv=kv)


@pytest.mark.parametrize("q,kv", TYPES)
@pytest.mark.parametrize("table", [0, FAR])
def test_the_same_call_gives_the_same(q, kv, table):
    """Bit for bit, whatever the workspace holds: with few pairs, in tiles, and in tiles side by side."""
    for rows, lens, heads, kv_heads in (([26], [1500], 8, 2), ([40, 9, 64], [300, 2000, 700], 8, 2), ([128, 1], [3000, 500], 8, 1)):
        c = B.PagedCase(rows, lens, heads, kv_heads, 128, 64, q, kv, seed=1)
        widen(c, table, 64)
        masks = torch.cat([T.bits(s, 2) for s in trees(rows)] + [torch.zeros(3, 2, dtype=torch.int64)]).cuda()
        pages = binding.Pages(c.k_pages, c.v_pages)
        ws = binding.paged_attention_workspace(pages, heads, q)
        first = None
        for fill in (0, 1, 127, 255):
            ws.fill_(fill)
            got = binding.knnssd_tree_attention(pages, c.block_table, c.row_start, c.kv_len, masks, c.q, ws, out=torch.zeros_like(c.q))
            first = got if first is None else first
            assert torch.equal(got, first)
