"""Row starts that lie: entries at the ends of 32 bits, and in any order."""
import math

import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
LOW, TOP = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16), (F32, F32)], ids=["bf16", "fp32_bf16", "fp32"])
@pytest.mark.parametrize("rows,lens", [([3, 40], [100, 90]), ([3, 2], [900, 700])])
def test_starts_from_end_to_end_of_32_bits(rows, lens, types):
    """What lies around the batch's rows of queries and outputs is neither written nor seen, and the call after it is as before."""
    c = B.PagedCase(rows, lens, 4, 2, 64, 16, *types)
    n, most = c.q.shape[0], max(rows)
    room = torch.full((3 * n, 4, 64), 7.0, dtype=types[0], device="cuda")
    out = room[n:2 * n]
    seen = torch.full((3 * n, 4, 64), math.nan, dtype=types[0], device="cuda")
    q = seen[n:2 * n]
    q.copy_(c.q)
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, 4, types[0])

    def run(most_rows):
        binding.knnssd_paged_attention(pages, c.block_table, c.row_start, c.kv_len, q, ws, out=out, most_rows=most_rows)

    out.fill_(5.0)
    run(most)
    good, start = out.clone(), c.row_start.clone()
    for bad in ([TOP, -9, 43], [5, LOW, 43], [0, 5, LOW], [LOW, TOP, LOW], [TOP, LOW, TOP], [LOW, LOW, TOP], [TOP, TOP, TOP], [n, TOP, LOW]):
        c.row_start.copy_(torch.tensor(bad, dtype=torch.int32))
        for m in (0, most):
            run(m)
        if types[0] == types[1]:
            binding.knnssd_prompt_attention(q, q[:, :2], q[:, 2:], c.row_start, out=out)
        torch.cuda.synchronize()
        assert (room[:n] == 7).all() and (room[2 * n:] == 7).all(), bad
    c.row_start.copy_(start)
    out.fill_(5.0)
    run(most)
    assert torch.equal(out, good)
