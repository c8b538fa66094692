"""Attention over pages and over packed prompts against the definition in 64 bits."""
import math

import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]
IDS = ["bf16", "fp32_bf16", "fp32"]


def run_paged(c, ws=None, scale=None, most_rows=0, **kw):
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, c.heads, c.q.dtype) if ws is None else ws
    return binding.knnssd_paged_attention(pages, c.block_table, c.row_start, c.kv_len, c.q, ws, out=c.out, scale=scale, most_rows=most_rows, **kw)


def check_paged(c, scale=None, most_rows=0, ws=None):
    want, err = c.want(c.dim ** -0.5 if scale is None else scale, BF16 if c.q.dtype == BF16 else None)
    B.check_rows(run_paged(c, ws, scale, most_rows), want, err, c.q.dtype)


FEW = [  # rows, lengths
    ([1], [1]), ([1], [2]), ([1], [64]), ([1], [65]), ([1], [255]), ([1], [257]), ([2], [1000]), ([1, 0, 3, 1], [5, 0, 3, 40]), ([5, 1, 9, 4, 16], [700, 31, 300, 129, 16]),
    ([3, 2, 2], [1, 0, 5]),          # rows whose positions lie before the request's first: nothing to see
    ([0, 0, 2, 0], [100, 0, 70, 9]), ([1] * 40, list(range(1, 200, 5)))]


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (5, 1, 128), (6, 2, 64), (8, 8, 128), (16, 1, 64)])
@pytest.mark.parametrize("which", range(len(FEW)))
def test_few_rows(which, heads, kv_heads, dim, types):
    rows, lens = FEW[which]
    check_paged(B.PagedCase(rows, lens, heads, kv_heads, dim, 16, *types, seed=which), most_rows=max(rows))


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("page,order", [(8, "head"), (8, "position"), (64, "position"), (256, "head"), (1024, "position")])
def test_pages_and_orders(page, order, types):
    check_paged(B.PagedCase([3, 1, 20], [page * 3 + 1, page, page + 19], 6, 3, 128, page, *types, order=order, gap=2), most_rows=20)
    check_paged(B.PagedCase([2, 70], [9, 2 * page + 71], 4, 2, 64, page, *types, order=order, gap=1))


MANY = [([17], [17]), ([33, 1, 65], [33, 90, 300]), ([130], [131]), ([100, 3, 0, 64], [400, 3, 77, 64]), ([200], [199]), ([63, 5], [1, 5])]


@pytest.mark.parametrize("hint", [False, True])
@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 128), (5, 1, 64), (3, 1, 128)])
@pytest.mark.parametrize("which", range(len(MANY)))
def test_chunks(which, heads, kv_heads, dim, types, hint):
    rows, lens = MANY[which]
    check_paged(B.PagedCase(rows, lens, heads, kv_heads, dim, 32, *types, seed=which), most_rows=max(rows) if hint else 0)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_a_wrong_bound_of_rows_only_costs_time(types):
    check_paged(B.PagedCase([40, 1], [90, 50], 10, 2, 64, 16, *types), most_rows=1)
    check_paged(B.PagedCase([1, 1], [90, 50], 10, 2, 64, 16, *types), most_rows=100000)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(scale, types):
    """A scale of 1 makes the softmax nearly one-hot; 0 the mean of the values."""
    check_paged(B.PagedCase([3, 20], [300, 70], 4, 2, 64, 16, *types), scale=scale)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_scores_far_from_zero(types):
    """Scores around +-3000 and rising along the axis: the running maximum carries them."""
    c = B.PagedCase([2, 33], [600, 290], 4, 2, 64, 16, *types)
    for sign in (1, -1):
        c.q.fill_(sign * 2.0)
        for r in range(2):
            ramp = torch.linspace(100, 187, c.lens[r])[:, None, None].expand_as(c.k[r]).to(c.k[r].dtype)
            c.k[r] = ramp.contiguous()
            for j in range(-(-c.lens[r] // 16)):
                m = min(16, c.lens[r] - j * 16)
                c.k_pages[c.table[r, j], :, :m] = c.k[r][j * 16:j * 16 + m].permute(1, 0, 2).cuda()
        check_paged(c, scale=0.125)


def test_long_axis_few_rows():
    """20 000 positions, the last page ending inside a tile; a table of one request of many."""
    check_paged(B.PagedCase([5, 1], [20011, 37], 5, 1, 128, 64, BF16, BF16), most_rows=5)
    check_paged(B.PagedCase([2, 1], [9001, 37], 2, 2, 64, 128, F32, BF16), most_rows=2)


def test_offsets_beyond_32_bits():
    """Pages of a pool of more than 2^32 elements: the last ones are read, not their remainders."""
    n_pages, page, dim = 1, 1024, 128
    stride = 2 ** 32 // 4 + 8 * 64
    buf = torch.empty(5 * stride + page * dim, dtype=BF16, device="cuda")
    k = buf.as_strided((6, 1, page, dim), (stride, page * dim, dim, 1))
    g = torch.Generator().manual_seed(3)
    kc, vc = (torch.randn(page, 1, dim, generator=g).to(BF16) for _ in range(2))
    v = torch.empty_like(buf).as_strided(k.shape, k.stride())
    k[5, 0], v[5, 0] = kc[:, 0].cuda(), vc[:, 0].cuda()
    pages = binding.Pages(k, v)
    for rows, most in ((2, 2), (200, 0)):
        q = torch.randn(rows, 2, dim, generator=g).to(BF16)
        out = binding.knnssd_paged_attention(pages, torch.tensor([[5]], dtype=torch.int32, device="cuda"), torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                                             torch.tensor([1000], dtype=torch.int32, device="cuda"), q.cuda(), binding.paged_attention_workspace(pages, 2, BF16),
                                             most_rows=most)
        want, err = B.attend64(q, kc[:1000], vc[:1000], dim ** -0.5, BF16)
        B.check_rows(out, want, err, BF16)
    assert n_pages == 1


PROMPTS = [[1], [2, 1], [16], [17, 0, 1], [63, 64, 65], [129, 5], [0, 0, 300, 0], [40] * 7, [255, 257]]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (4, 4, 128), (10, 2, 64), (3, 1, 128)])
@pytest.mark.parametrize("which", range(len(PROMPTS)))
def test_prompts(which, heads, kv_heads, dim, dtype):
    """Packed prompts, queries, keys and values parts of one row; rows behind the last prompt hold NaN and stay out of it."""
    lens = PROMPTS[which]
    g = torch.Generator().manual_seed(which)
    total, pad = sum(lens), 5
    qkv = torch.randn(total + pad, heads + 2 * kv_heads, dim, generator=g).to(dtype)
    qkv[total:] = math.nan
    out = torch.full((total + pad, heads, dim), 5.0, dtype=dtype, device="cuda")
    start = [0]
    for a in lens:
        start.append(start[-1] + a)
    x = qkv.cuda()
    q, k, v = x.split([heads, kv_heads, kv_heads], 1)
    binding.knnssd_prompt_attention(q, k, v, torch.tensor(start, dtype=torch.int32, device="cuda"), out=out)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    both = [B.attend64(q[a:b], k[a:b], v[a:b], dim ** -0.5, BF16 if dtype == BF16 else None) for a, b in zip(start, start[1:])]
    B.check_rows(out, torch.cat([o for o, _ in both]), torch.cat([e for _, e in both]), dtype)


def test_the_same_call_has_the_same_bits_and_leaves_the_workspace_ready():
    """One workspace over batches of several shapes, in turn; every repetition has the bits of the first."""
    cases = [B.PagedCase([2, 1, 5], [900, 3000, 41], 8, 2, 128, 32, BF16, BF16, seed=1), B.PagedCase([1], [5000], 8, 2, 128, 32, BF16, BF16, seed=2),
             B.PagedCase([70, 1], [800, 700], 8, 2, 128, 32, BF16, BF16, seed=3)]
    ws = binding.paged_attention_workspace(binding.Pages(cases[0].k_pages, cases[0].v_pages), 8, BF16)
    first = [run_paged(c, ws).clone() for c in cases]
    for _ in range(5):
        for c, f in zip(cases, first):
            c.out.fill_(5.0)
            assert torch.equal(run_paged(c, ws), f)
    for c in cases:
        check_paged(c, ws=ws)


def test_in_a_graph_with_lengths_that_change():
    """A captured step is replayed with other lengths and tables; eager calls with the same workspace in between."""
    c = B.PagedCase([4, 3, 1], [2000, 310, 77], 8, 2, 64, 16, BF16, BF16)
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, 8, BF16)
    run_paged(c, ws)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:        # two graphs that share the workspace
        with torch.cuda.graph(g):
            run_paged(c, ws)
    full = list(c.lens)
    for i, lens in enumerate(([2000, 310, 77], [3, 3, 1], [1999, 1, 0], [700, 300, 60], [2000, 310, 77])):
        c.lens = lens
        c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        c.out.fill_(5.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = c.out.clone()
        keep = c.k, c.v
        c.k, c.v = [t[:n] for t, n in zip(c.k, lens)], [t[:n] for t, n in zip(c.v, lens)]
        want, err = c.want(0.125, BF16)
        B.check_rows(got, want, err, BF16)
        assert torch.equal(run_paged(c, ws), got)
        c.k, c.v = keep
    assert full == c.lens


def test_two_streams():
    """Two batches at once, a workspace each, on streams that are not the tensors' own."""
    cases = [B.PagedCase([3, 1], [4000, 900], 8, 2, 128, 32, BF16, BF16, seed=s) for s in (1, 2)]
    streams = [torch.cuda.Stream() for _ in cases]
    work = [binding.paged_attention_workspace(binding.Pages(c.k_pages, c.v_pages), 8, BF16) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, w in zip(cases, streams, work):
            run_paged(c, w, stream=s)
    torch.cuda.synchronize()
    for c in cases:
        want, err = c.want(c.dim ** -0.5, BF16)
        B.check_rows(c.out, want, err, BF16)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_values_that_are_not_finite_in_places_that_no_row_sees(types):
    """A request of no rows whose cache holds NaN, page tails and pages of nobody (NaN in every case here), and a table whose ids lie outside the cache."""
    c = B.PagedCase([2, 0, 1], [40, 60, 33], 4, 2, 64, 16, *types)
    for j in range(4):
        c.k_pages[c.table[1, j]] = math.nan
        c.v_pages[c.table[1, j]] = math.inf
    check_paged(c)
    check_paged(c, most_rows=100)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,lens", [([3, 1, 2], [900, 40, 700]), ([60, 30], [900, 200]), ([2, 3], [30, 40])])
def test_not_a_number_stays_in_the_rows_that_see_it(rows, lens, types):
    """A query, and a key that all rows of a request see: their outputs are NaN, all others as without."""
    c = B.PagedCase(rows, lens, 4, 2, 64, 16, *types)
    good = run_paged(c, most_rows=max(rows)).clone()
    c.q[0, 1] = math.nan                                      # row 0, head 1
    c.k_pages[c.table[1, 0], 1, 3] = math.nan                 # request 1, kv head 1
    c.out.fill_(5.0)
    got = run_paged(c, most_rows=max(rows))
    lost = torch.zeros(got.shape[:2], dtype=torch.bool)
    lost[0, 1] = True
    lost[c.start[1]:c.start[2], 2:] = True
    assert torch.isnan(got[lost]).all()
    assert torch.equal(got[~lost], good[~lost])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [[5, 9], [300, 170]])
def test_not_a_number_in_a_prompt(rows, dtype):
    """A query's is its own row's; a key's is that of its own row and the later ones of its request."""
    g = torch.Generator().manual_seed(9)
    start = torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn(sum(rows), h, 64, generator=g).to(dtype).cuda() for h in (4, 2, 2))
    good = binding.knnssd_prompt_attention(q, k, v, start).clone()
    q[1, 1] = math.nan
    k[rows[0] + 4, 1] = math.nan
    got = binding.knnssd_prompt_attention(q, k, v, start)
    lost = torch.zeros(got.shape[:2], dtype=torch.bool)
    lost[1, 1] = True
    lost[rows[0] + 4:, 2:] = True
    assert torch.isnan(got[lost]).all()
    assert torch.equal(got[~lost], good[~lost])


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_tables_that_lie_point_somewhere_in_the_cache(types):
    """Page ids outside the cache, lengths beyond the table, rows beyond the batch: wrong values, never an access out of range."""
    c = B.PagedCase([3, 40], [100, 90], 4, 2, 64, 16, *types)
    good = run_paged(c, most_rows=40).clone()
    table, lens, start = c.block_table.clone(), c.kv_len.clone(), c.row_start.clone()
    for bad in (-1, 2 ** 31 - 1, -2 ** 31, c.k_pages.shape[0]):
        c.block_table[0].fill_(bad)
        run_paged(c)
    c.block_table.copy_(table)
    for bad in (2 ** 31 - 1, -5, -2 ** 31):
        c.kv_len[0] = bad
        run_paged(c)
    c.kv_len.copy_(lens)
    for bad in ([0, 2 ** 31 - 1, 43], [0, 3, 2 ** 31 - 1], [-7, 3, 43], [5, 3, 43], [0, -9, 43], [0, 0, 0]):
        c.row_start.copy_(torch.tensor(bad, dtype=torch.int32))
        run_paged(c)
        binding.knnssd_prompt_attention(c.q, c.q[:, :2], c.q[:, 2:], c.row_start, out=c.out)
    c.row_start.copy_(start)
    c.out.fill_(5.0)
    assert torch.equal(run_paged(c, most_rows=40), good)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_many_requests(types):
    """More requests than a wavefront looks at once (64), most of them without rows."""
    rows = [0] * 300
    for i, n in ((0, 2), (63, 1), (64, 3), (130, 20), (299, 1)):
        rows[i] = n
    lens = [r + (7 * i) % 50 for i, r in enumerate(rows)]
    c = B.PagedCase(rows, lens, 4, 2, 64, 8, *types)
    check_paged(c, most_rows=3 if types[0] == F32 else 0)
    check_paged(c, most_rows=20)


def test_scores_that_leave_the_first_block_far_behind():
    """Tiles weigh against the first block's largest score: later ones 2^64 and more above it make the reference follow, in rows of their own."""
    c = B.PagedCase([40, 3], [500, 200], 4, 2, 64, 16, BF16, BF16)
    for r in range(2):
        up = torch.ones(c.lens[r], 1, 1)
        up[70:] = 40.0                                        # scores up to 40 times as large from here on, and again behind 300
        up[300:] = 400.0
        c.k[r] = (c.k[r].float() * up).to(BF16)
        for j in range(-(-c.lens[r] // 16)):
            m = min(16, c.lens[r] - j * 16)
            c.k_pages[c.table[r, j], :, :m] = c.k[r][j * 16:j * 16 + m].permute(1, 0, 2).cuda()
    check_paged(c)
    check_paged(c, scale=1.0)


@pytest.mark.parametrize("heads,kv_heads,dim", [(40, 40, 128), (10, 2, 64), (8, 8, 64)])
def test_fp32_on_the_matrix_cores(heads, kv_heads, dim):
    """Enough rows, or a long enough table, for the tiles in fp32: prompts, chunks and single rows."""
    check_paged(B.PagedCase([120, 1, 300 if dim == 64 else 30], [500, 2300, 301], heads, kv_heads, dim, 32, F32, F32), most_rows=300)
    check_paged(B.PagedCase([1, 5], [2500, 70], heads, kv_heads, dim, 16, F32, F32, order="position"), most_rows=5)
    g = torch.Generator().manual_seed(dim)
    lens = [0, 130, 1, 300 if dim == 64 else 64, 33]
    start = [sum(lens[:i]) for i in range(len(lens) + 1)]
    qkv = torch.randn(start[-1] + 60, heads + 2 * kv_heads, dim, generator=g)
    qkv[start[-1]:] = math.nan
    n_rows = max(qkv.shape[0], 4200 // heads)
    qkv = torch.cat([qkv, torch.full((n_rows - qkv.shape[0] + 1, *qkv.shape[1:]), math.nan)])
    out = torch.full((qkv.shape[0], heads, dim), 5.0, device="cuda")
    q, k, v = qkv.cuda().split([heads, kv_heads, kv_heads], 1)
    binding.knnssd_prompt_attention(q, k, v, torch.tensor(start, dtype=torch.int32, device="cuda"), out=out)
    q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
    both = [B.attend64(q[a:b], k[a:b], v[a:b], dim ** -0.5) for a, b in zip(start, start[1:])]
    B.check_rows(out, torch.cat([o for o, _ in both]), torch.cat([e for _, e in both]), F32)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("dim", [64, 128])
def test_a_group_of_more_heads_than_a_tile_has_pairs(dim, types):
    """200 query heads of one kv head: a row's heads lie in two or three tiles, 13 groups of 16."""
    check_paged(B.PagedCase([2, 0, 3, 1], [70, 5, 3, 300], 200, 1, dim, 16, *types))
    check_paged(B.PagedCase([1], [90], 200, 1, dim, 16, *types), most_rows=1)
    if types[0] == types[1]:
        g = torch.Generator().manual_seed(3)
        q, k, v = (torch.randn(35, h, dim, generator=g).to(types[0]) for h in (200, 1, 1))
        out = binding.knnssd_prompt_attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, 2, 35], dtype=torch.int32, device="cuda"))
        both = [B.attend64(q[a:b], k[a:b], v[a:b], dim ** -0.5, BF16 if types[0] == BF16 else None) for a, b in ((0, 2), (2, 35))]
        B.check_rows(out, torch.cat([o for o, _ in both]), torch.cat([e for _, e in both]), types[0])


@pytest.mark.parametrize("types", TYPES, ids=IDS)
def test_the_most_requests_of_a_call(types):
    """4096 requests, over pages with and without a bound of their rows, and as prompts of no row or one."""
    rows = [1] * 4090 + [0, 0, 2, 0, 0, 3]
    lens = [a + (7 * i) % 30 for i, a in enumerate(rows)]
    c = B.PagedCase(rows, lens, 2, 1, 64, 8, *types)
    want, err = c.want(0.125, BF16 if types[0] == BF16 else None)
    for most in (3, 0):
        c.out.fill_(5.0)
        B.check_rows(run_paged(c, most_rows=most), want, err, types[0])
    if types[0] == types[1]:
        out = binding.knnssd_prompt_attention(c.q[:4090], c.q[:4090, :1], c.q[:4090, 1:], c.row_start)
        # One row a request: its own value v, as (w v) (1 / w) with a weight w that the score's product and sum leave within some steps of 1. Three
        # roundings, the product's, the reciprocal's and their product's, of half a step each: (1 + e)^3 - 1 < 4 e. Rounded to bf16 that is v.
        own = c.q[:4090, 1:].expand(-1, 2, -1)
        assert ((out - own).abs() <= (0 if types[0] == BF16 else 4 * B.EPS32) * own.abs()).all()
