"""Results that the batch calls allocate themselves, on a stream that is not the current one."""
import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def calls():
    """(a call that makes its own output on a stream, what it gives, the error allowed) for attention over pages and over prompts."""
    c = B.PagedCase([40, 3], [90, 700], 8, 2, 64, 16, BF16, BF16, pad=0)
    pages = binding.Pages(c.k_pages, c.v_pages)
    ws = binding.paged_attention_workspace(pages, 8, BF16)
    want, err = c.want(0.125, BF16)
    yield lambda s: binding.knnssd_paged_attention(pages, c.block_table, c.row_start, c.kv_len, c.q, ws, stream=s), want, err
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(43, h, 64, generator=g).to(BF16) for h in (8, 2, 2))
    on = [t.cuda() for t in (q, k, v)]
    start = torch.tensor([0, 43], dtype=torch.int32, device="cuda")
    want, err = B.attend64(q, k, v, 0.125, BF16)
    yield lambda s: binding.knnssd_prompt_attention(*on, start, stream=s), want, err


def busy(a, b):
    for _ in range(20):
        torch.mm(a, a, out=b)


def test_memory_that_the_current_stream_still_writes_is_not_the_result():
    """The host has given back a block of the result's size that the current stream has yet to write."""
    a = torch.randn(4096, 4096, device="cuda")
    b = torch.empty_like(a)
    for call, want, err in calls():
        stream = torch.cuda.Stream()
        busy(a, b)
        torch.cuda.synchronize()
        busy(a, b)
        block = torch.empty(43, 8, 64, dtype=BF16, device="cuda")
        at = block.data_ptr()
        block.fill_(7.0)
        del block
        out = call(stream)
        assert out.data_ptr() != at
        torch.cuda.synchronize()
        B.check_rows(out, want, err, BF16)


def test_a_result_that_the_current_stream_still_reads_is_not_the_next_one():
    a = torch.randn(4096, 4096, device="cuda")
    b = torch.empty_like(a)
    for call, want, err in calls():
        stream = torch.cuda.Stream()
        copy = torch.empty(43, 8, 64, dtype=BF16, device="cuda")
        busy(a, b)
        torch.cuda.synchronize()
        out = call(stream)
        torch.cuda.current_stream().wait_stream(stream)
        busy(a, b)
        copy.copy_(out)
        at = out.data_ptr()
        del out
        out = call(stream)
        assert out.data_ptr() != at
        torch.cuda.synchronize()
        B.check_rows(copy, want, err, BF16)


def test_a_result_on_the_current_stream():
    for call, want, err in calls():
        for stream in (None, torch.cuda.current_stream()):
            B.check_rows(call(stream), want, err, BF16)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            out = call(None)
        stream.synchronize()
        B.check_rows(out, want, err, BF16)


def test_a_result_on_a_stream_forked_from_a_captured_one():
    """Several replays, with eager calls in between."""
    for call, want, err in calls():
        side = torch.cuda.Stream()
        eager = call(None)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            current = torch.cuda.current_stream()
            side.wait_stream(current)
            out = call(side)
            current.wait_stream(side)
        for _ in range(4):
            out.fill_(5.0)
            graph.replay()
            torch.cuda.synchronize()
            B.check_rows(out, want, err, BF16)
            assert torch.equal(call(None), eager) and torch.equal(out, eager)
