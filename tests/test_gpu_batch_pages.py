"""Page plans and the rotary store into pages, against plain forms (lists; 64 bits)."""
import math
import random

import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def state(t):
    return dict(table=t.block_table.tolist(), held=t.held.tolist(), free=t.free_pages[:t.n_free.item()].tolist())


def same(stack, tables, want, rows):
    for name in ("row_start", "kv_len", "slots", "positions", "result"):
        assert getattr(rows, name).tolist() == want[name], name
    got = state(tables)
    assert got["held"] == stack.held and got["free"] == stack.free
    assert got["table"] == stack.table


@pytest.mark.parametrize("n,page,most,max_rows", [(1, 8, 3, 40), (3, 16, 40, 200), (64, 64, 9, 700), (65, 32, 300, 25000), (1000, 8, 5, 5000), (4096, 16, 2, 9000)])
def test_rounds_of_a_batch(n, page, most, max_rows):
    """Rounds with rows tried, rows kept, requests that end and begin again: tables, stack and slots as the lists have them."""
    rng = random.Random(n)
    longest = 6 * most + 40
    pages = sum(-(-longest // page) for _ in range(n))
    stack = B.Stack(n, -(-longest // page), pages, page)
    tables = binding.PageTables.fresh(n, longest, pages, page)
    rows = binding.BatchRows(n, max_rows)
    cached = [0] * n
    for _ in range(5):
        added = [rng.randint(0, most) for _ in range(n)]
        want = stack.plan(cached, added, max_rows)
        binding.knnssd_page_plan(tables, rows, ints(cached), ints(added))
        same(stack, tables, want, rows)
        assert want["result"][2] == 0
        assert len(set(s for s in want["slots"] if s >= 0)) == sum(added)
        cached = [0 if rng.random() < 0.2 else c + rng.randint(0, a) for c, a in zip(cached, added)]


@pytest.mark.parametrize("n,max_rows", [(5, 100), (300, 1500), (2000, 9000)])
def test_lengths_over_the_arrays_of_the_last_round(n, max_rows):
    """cached (then added) is the round's own kv_len: the plan overwrites its own argument."""
    rng = random.Random(n)
    stack, tables, rows = B.Stack(n, 8, 6 * n, 8), binding.PageTables.fresh(n, 64, 6 * n, 8), binding.BatchRows(n, max_rows)
    cached = [0] * n
    rows.kv_len.zero_()
    for _ in range(8):
        added = [rng.randint(0, 4) for _ in range(n)]
        want = stack.plan(cached, added, max_rows)
        binding.knnssd_page_plan(tables, rows, rows.kv_len, ints(added))
        same(stack, tables, want, rows)
        cached = want["kv_len"]
    added = [rng.randint(0, 4) for _ in range(n)]
    rows.kv_len.copy_(ints(added))
    want = stack.plan([9] * n, added, max_rows)
    binding.knnssd_page_plan(tables, rows, ints([9] * n), rows.kv_len)
    same(stack, tables, want, rows)


def test_the_largest_batch_whose_last_request_has_all_rows():
    n = 4096
    stack, tables, rows = B.Stack(n, 5, 9, 8), binding.PageTables.fresh(n, 40, 9, 8), binding.BatchRows(n, 40)
    added = [0] * (n - 1) + [37]
    want = stack.plan([0] * n, added, 40)
    binding.knnssd_page_plan(tables, rows, ints([0] * n), ints(added))
    same(stack, tables, want, rows)


@pytest.mark.parametrize("max_rows", [50, 5000])
@pytest.mark.parametrize("cached,added,flag", [
    ([5, -1, 0], [1, 1, 1], 1), ([5, 0, 0], [1, -2, 1], 1), ([2 ** 31 - 1, 0, 0], [2 ** 31 - 1, 0, 0], 1),
    ([0, 0, 0], [4000, 2000, 1], 2), ([0, 0, 0], [2 ** 31 - 1, 2 ** 31 - 1, 5], 2), ([30, 0, 0], [11, 0, 0], 3), ([30, 30, 30], [1, 1, 1], 4)])
def test_a_plan_that_cannot_be_done_changes_nothing(cached, added, flag, max_rows):
    stack, tables, rows = B.Stack(3, 5, 11, 8), binding.PageTables.fresh(3, 40, 11, 8), binding.BatchRows(3, max_rows)
    for c, a in (([0, 0, 0], [9, 8, 1]),):
        want = stack.plan(c, a, max_rows)
        binding.knnssd_page_plan(tables, rows, ints(c), ints(a))
        same(stack, tables, want, rows)
    want = stack.plan(cached, added, max_rows) if flag != 1 else dict(row_start=[0] * 4, kv_len=[0] * 3, slots=[-1] * max_rows, positions=[-1] * max_rows, result=[0, 0, 1, 0])
    assert want["result"][2] == flag
    binding.knnssd_page_plan(tables, rows, ints(cached), ints(added))
    same(stack, tables, want, rows)


@pytest.mark.parametrize("spoil", [dict(held=[2, -1, 1]), dict(held=[2, 6, 1]), dict(n_free=-1), dict(n_free=12), dict(n_free=11)])
def test_malformed_tables_are_told(spoil):
    """held or n_free outside what the tables can hold, and more pages given back than the pool has."""
    tables, rows = binding.PageTables.fresh(3, 40, 11, 8), binding.BatchRows(3, 20)
    binding.knnssd_page_plan(tables, rows, ints([0, 0, 0]), ints([9, 8, 1]))
    if "held" in spoil:
        tables.held.copy_(ints(spoil["held"]))
    else:
        tables.n_free.fill_(spoil["n_free"])
    before = state(tables) if spoil.get("n_free", 0) >= 0 and spoil.get("n_free", 0) <= 11 else None
    binding.knnssd_page_plan(tables, rows, ints([0, 0, 0]), ints([0, 0, 0]))
    assert rows.result.tolist() == [0, 0, 1, 0]
    assert before is None or state(tables) == before


STORE = [  # heads, kv heads, dim, page, rows dtype, cache dtype
    (4, 4, 64, 16, "fp32", "fp32"), (40, 8, 128, 64, "bf16", "bf16"), (5, 1, 128, 8, "fp32", "bf16"), (0, 3, 64, 32, "bf16", "bf16"), (9, 9, 128, 1024, "bf16", "bf16")]
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("order", ["head", "position"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,qt,kt", STORE)
def test_store(heads, kv_heads, dim, page, qt, kt, order):
    """Odd positions up to 2^31 - 1, skipped rows, strided rows; untouched places keep what they had, values arrive bit for bit."""
    g = torch.Generator().manual_seed(heads + dim)
    n_pages, n, base = 7, 13, 500000.0
    qkv = torch.randn(n, (heads + 2 * kv_heads) * dim + 8, generator=g).to(DT[qt]).cuda()[:, :-8]
    shape = (n_pages, kv_heads, page, dim) if order == "head" else (n_pages, page, kv_heads, dim)
    turn = (0, 1, 2, 3) if order == "head" else (0, 2, 1, 3)
    k, v = (torch.full(shape, 3.0, dtype=DT[kt], device="cuda").permute(turn) for _ in range(2))
    slots = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
    positions = torch.tensor([0, 1, 2, 7, 63, 1000, 4095, 65537, 131072, 1000003, 2 ** 31 - 1, 12, 13], dtype=torch.int32)
    slots[3], slots[8], positions[5] = -1, n_pages * page, -1
    live = [i for i in range(n) if i not in (3, 8, 5)]
    q_out = torch.full((n, heads + 1, dim), 9.0, dtype=DT[qt], device="cuda")[:, :heads] if heads else None
    k_out = torch.full((n, kv_heads, dim), 9.0, dtype=DT[qt], device="cuda")
    binding.knnssd_paged_store(binding.Pages(k, v), qkv, slots.cuda(), positions.cuda(), base, q_out, k_out)
    x = qkv.cpu().double().view(n, heads + 2 * kv_heads, dim)
    i = torch.arange(dim // 2, dtype=torch.float64)
    angle = positions.double()[:, None] * base ** (-2 * i / dim)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    # sine and cosine of angles in turns, half a turn at most: the rest's rounding (half a step of a value up to 1, in half turns) and the
    # functions' own four half steps; two products and a sum of half a step each. Angles in 64 bits: 2^31 radians are off by 2^31 2^-53 2 pi at most,
    # a few times over.
    size = torch.cat([a.abs() + b.abs(), a.abs() + b.abs()], -1)
    slack = size * (math.pi * B.EPS32 + 7 * B.EPS32 + 2 ** 31 * 2.0 ** -53 * 40)

    def near(got, want, err, dtype):
        got = got.cpu().double()
        assert ((got - want).abs() <= err + B.half_step(dtype) * (want.abs() + err)).all()

    if heads:
        near(q_out[live], turned[live, :heads], slack[live, :heads], DT[qt])
        assert (q_out[[3, 5, 8]] == 9).all()
    near(k_out[live], turned[live, heads:heads + kv_heads], slack[live, heads:heads + kv_heads], DT[qt])
    assert (k_out[[3, 5, 8]] == 9).all()
    want_k, want_v = torch.full(k.shape, 3.0).double(), torch.full(k.shape, 3.0, dtype=DT[kt])
    err_k = torch.zeros(k.shape).double()
    for r in live:
        at = slots[r].item()
        want_k[at // page, :, at % page] = turned[r, heads:heads + kv_heads]
        err_k[at // page, :, at % page] = slack[r, heads:heads + kv_heads]
        want_v[at // page, :, at % page] = qkv[r].cpu().view(-1, dim)[heads + kv_heads:].to(DT[kt])
    near(k, want_k, err_k, DT[kt])
    assert torch.equal(v.cpu(), want_v)


def test_store_in_place_and_non_finite_values():
    """q_out and k_out over the same heads of qkv; infinities and NaN of values pass through."""
    n, heads, kv_heads, dim = 5, 6, 2, 64
    qkv = torch.randn(n, (heads + 2 * kv_heads) * dim, device="cuda").bfloat16()
    x = qkv.view(n, -1, dim)
    x[1, heads + kv_heads, 3], x[2, heads + kv_heads, 5], x[3, -1, -1] = math.inf, math.nan, -math.inf
    other, q_out, k_out = qkv.clone(), torch.empty(n, heads, dim, device="cuda").bfloat16(), torch.empty(n, kv_heads, dim, device="cuda").bfloat16()
    pages = [binding.Pages.empty(2, 8, kv_heads, dim) for _ in range(2)]
    slots, positions = ints([3, 1, 9, 15, 0]), ints([4, 99, 3, 0, 7])
    for p in pages:
        p.k.zero_(), p.v.zero_()
    binding.knnssd_paged_store(pages[0], other, slots, positions, q_out=q_out, k_out=k_out)
    assert torch.equal(other.view(torch.int16), qkv.view(torch.int16))
    x = other.view(n, -1, dim)
    binding.knnssd_paged_store(pages[1], other, slots, positions, q_out=x[:, :heads], k_out=x[:, heads:heads + kv_heads])
    assert torch.equal(x[:, :heads], q_out) and torch.equal(x[:, heads:heads + kv_heads], k_out)
    assert torch.equal(pages[0].k, pages[1].k) and torch.equal(pages[0].v.view(torch.int16), pages[1].v.view(torch.int16))
    got = pages[0].v
    assert got[0, 0, 1, 3] == math.inf and math.isnan(got[1, 0, 1, 5].item()) and got[1, 1, 7, 63] == -math.inf


def test_plan_and_store_in_a_graph():
    """A captured round follows the lengths that are written between its replays."""
    n, page, max_rows, dim = 3, 8, 30, 64
    tables, rows = binding.PageTables.fresh(n, 80, 30, page), binding.BatchRows(n, max_rows)
    stack = B.Stack(n, 10, 30, page)
    pages = binding.Pages.empty(30, page, 2, dim)
    qkv = torch.randn(max_rows, 5 * dim, device="cuda").bfloat16()
    q_out = torch.zeros(max_rows, 1, dim, device="cuda").bfloat16()
    cached, added = ints([0] * n), ints([0] * n)

    def step():
        binding.knnssd_page_plan(tables, rows, cached, added)
        binding.knnssd_paged_store(pages, qkv, rows.slots, rows.positions, q_out=q_out)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for c, a in (([0, 0, 0], [7, 9, 1]), ([7, 9, 1], [1, 8, 8]), ([8, 10, 0], [1, 1, 0]), ([0, 11, 0], [20, 1, 3])):
        cached.copy_(ints(c)), added.copy_(ints(a))
        pages.v.zero_()
        graph.replay()
        want = stack.plan(c, a, max_rows)
        same(stack, tables, want, rows)
        for t, s in enumerate(want["slots"]):
            if s >= 0:
                assert torch.equal(pages.v[s // page, :, s % page], qkv[t].view(5, dim)[3:])
        assert int((pages.v != 0).any(-1).any(1).sum()) == sum(a)
