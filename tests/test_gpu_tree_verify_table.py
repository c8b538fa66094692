"""knnssd_tree_verify in bf16 where the batch is so large that the rows' sums are taken by a table of powers (8192 chunks of 2048 tokens, of the rows that the arrays have): against the
plain form, on the CPU in 64 bits. Whole numbers: all have to be equal."""
import math

import pytest
import torch

import tree_common as T
from test_gpu_tree_verify import check, call

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def case(rows, vocab, drawn, **kw):
    """A case whose arrays have enough rows behind the last request's."""
    chunks = -(-vocab // 2048) * (2 if drawn else 1)
    need = max(8192, 64 * len(rows))
    return T.VerifyCase(rows, vocab, BF16, drawn, pad=max(2, -(-need // chunks) - sum(rows)), **kw)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab,gap", [(2047, 1), (2048, 0), (2049, 3), (5001, 0), (32000, 8), (70001, 0)])
def test_sizes(drawn, vocab, gap):
    check(case([1, 9, 0, 14, 5], vocab, drawn, temperatures=(0.8, 0.0, 1.3), gap=gap, seed=vocab))
    check(case([6, 2], vocab, drawn, shape="chain", temperatures=(0.5,), gap=gap, seed=vocab + 1), most_children=1)


@pytest.mark.parametrize("drawn", [False, True])
def test_many_rows_and_requests(drawn):
    check(case([1024, 300, 65], 4500, drawn, shape="tree", seed=1))
    check(case([(i * 7) % 5 for i in range(120)], 2100, drawn, shape="tree", temperatures=(0.9, 0.0, 2.0), seed=4))
    check(case([1], 40000, drawn, seed=5))


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("temperature", [0.01, 0.3, 1.0, 40.0, 1e38])
def test_values_at_the_ends_of_the_table(drawn, temperature):
    """The smallest and the largest values that it has and those beside them, none at all, and rows that lie far from 0."""
    ends = [0.0, -0.0, 2.0 ** -17, -2.0 ** -17, 2.0 ** -18, -2.0 ** -18, 1e-30, -1e-40, 255.0, -255.0, 256.0, -256.0, 300.0, -300.0, -5000.0, -3e38, -math.inf]
    rows = [2] * len(ends) + [3] * 6
    c = case(rows, 4100, drawn, shape="chain", temperatures=(temperature,), seed=3)
    for i, value in enumerate(ends):
        for row in (c.start[i], c.start[i] + 1):
            for at in (1, 777, 2047, 2048, 4099):             # (both chunks, the last of 52 tokens too)
                c.logits[row, at] = value
                if drawn and row == c.start[i]:
                    c.draft[row, at] = value
    for i, shift in enumerate((-300.0, -200.0, 200.0, 3000.0, -1e30, -math.inf)):
        row = c.start[len(ends) + i]
        if math.isinf(shift):
            c.logits[row, :2048] = shift                      # (a chunk of nothing)
        else:
            c.logits[row] = c.logits[row] + shift
    check(c)


@pytest.mark.parametrize("value", [math.nan, -math.nan, math.inf])
def test_values_that_are_no_numbers(value):
    for drawn in (False, True):
        c = case([1, 3, 3, 2], 4100, drawn, shape="chain", seed=6)
        for r, at in ((0, 0), (1, 2048), (2, 4099)):
            c.logits[c.start[r], at] = value
        if drawn:
            c.draft[c.start[3], 7] = value
        want = check(c)
        assert want[2][:3] == [-1, -1, -1] and (not drawn or want[2][3] == -1)


def test_the_same_call_gives_the_same():
    c = case([20, 8, 33], 30000, True, temperatures=(0.7, 1.1), seed=8)
    args = c.on_gpu()
    first = call(args, c.cap, 3, c.vocab)
    for fill in (0, 255, 127):
        assert all(torch.equal(a[:61], b[:61]) for a, b in zip(first, call(args, c.cap, 3, c.vocab, fill=fill)))


def test_row_starts_that_are_wrong():
    """Whatever they say, no row outside the batch is touched."""
    c = case([20, 8, 33], 5000, True, seed=9)
    args = c.on_gpu()
    for start in ([0, -5, 2 ** 31 - 1, 61], [7, 3, 50, 2 ** 31 - 1], [-2 ** 31, 61, 20, 28], [0, 0, 0, 0]):
        args["row_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        path = torch.full((c.cap + 64,), -9, dtype=torch.int32, device="cuda")
        call(args, c.cap, 3, c.vocab, path=path)
        assert (path[c.cap:] == -9).all()
