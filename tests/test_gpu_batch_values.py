"""Attention over pages and prompts where the values are large, or the scores far below what fp32 holds, in every kernel that a call may take."""
import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(BF16, BF16), (F32, BF16), (F32, F32)]
IDS = ["bf16", "fp32_bf16", "fp32"]
HEADS, KV, DIM, PAGE = 4, 2, 64, 16
FIRST = 64                              # no kernel takes more positions than these in its first block

# rows, lengths: one group of pairs and several, a request whose table is short enough for an fp32 cache's row kernel and ones that are not, axes that are
# split, down to a block each, and enough of them that every part has several blocks; prompts in one tile and in several
BATCHES = [([2], [300]), ([40, 3], [500, 200]), ([3] * 10, [9000] * 10), ([70, 2], [3000, 130]), ([200, 90], [200, 90]), ([700], [700])]


def outputs(q, k, v, types):
    """The batch over pages, with and without a bound of its rows, and (one type, a request's rows all of its positions) as prompts."""
    rows, lens = [a.shape[0] for a in q], [a.shape[0] for a in k]
    c = B.PagedCase(rows, lens, HEADS, KV, DIM, PAGE, *types)
    for r, n in enumerate(lens):
        for j in range(-(-n // PAGE)):
            m = min(PAGE, n - j * PAGE)
            for pages, t in ((c.k_pages, k[r]), (c.v_pages, v[r])):
                pages[c.table[r, j], :, :m] = t[j * PAGE:j * PAGE + m].permute(1, 0, 2).cuda()
    c.q[:sum(rows)] = torch.cat(q).cuda()
    pages = binding.Pages(c.k_pages, c.v_pages)
    for most in (0, max(rows)):
        c.out.fill_(5.0)
        yield binding.knnssd_paged_attention(pages, c.block_table, c.row_start, c.kv_len, c.q, binding.paged_attention_workspace(pages, HEADS, types[0]),
                                             out=c.out, most_rows=most)
    if types[0] == types[1] and rows == lens:
        out = torch.full_like(c.out, 5.0)
        yield binding.knnssd_prompt_attention(c.q, torch.cat(k + [k[0][:3]]).cuda(), torch.cat(v + [v[0][:3]]).cuda(), c.row_start, out=out)


def check(q, k, v, types, hidden=0):
    """Against the definition in 64 bits over the positions from `hidden` on; rows before that are not compared."""
    both = [B.attend64(a, b[hidden:], c[hidden:], DIM ** -0.5, BF16 if types[0] == BF16 else None) for a, b, c in zip(q, k, v)]
    want, err = (torch.cat(x) for x in zip(*both))
    seen = torch.cat([torch.arange(b.shape[0] - a.shape[0], b.shape[0]) >= hidden for a, b in zip(q, k)])
    for got in outputs(q, k, v, types):
        got = got.clone()
        got[:seen.numel()][~seen.cuda()] = 0          # (their definition over the compared positions is 0)
        B.check_rows(got, want, err, types[0])


def batch(rows, lens, types, level, values, g):
    """Queries of 2 in every dimension but for some noise, keys whose score with them is about level(position), values of `values` times a normal one."""
    q = [(2 + 0.01 * torch.randn(n, HEADS, DIM, generator=g)).to(types[0]) for n in rows]
    k = [(level(torch.arange(n, dtype=F32)) / 2 / DIM ** 0.5)[:, None, None].expand(n, KV, DIM).to(types[1]).contiguous() for n in lens]
    v = [(values * torch.randn(n, KV, DIM, generator=g)).to(types[1]) for n in lens]
    return q, k, v


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,lens", BATCHES)
def test_large_values_under_scores_that_rise(rows, lens, types):
    """Scores 0 in the first block and 38 (55 powers of two) behind it, values around 1e24: the outputs are as large as the values, and finite."""
    g = torch.Generator().manual_seed(1)
    check(*batch(rows, lens, types, lambda p: 38.0 * (p >= FIRST), 1e24, g), types)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("rows,lens", BATCHES)
def test_first_positions_whose_scores_fp32_does_not_hold(rows, lens, types):
    """Keys of -3e38 give the first block's positions scores of -inf: they have no weight, however far below zero the scores behind them are."""
    g = torch.Generator().manual_seed(2)
    q, k, v = batch(rows, lens, types, lambda p: -140.0 - (p % 5), 1.0, g)
    for t in k:
        t[:FIRST] = -3e38
    check(q, k, v, types, hidden=FIRST)
