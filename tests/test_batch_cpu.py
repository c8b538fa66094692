"""Refusals of the batch calls: every one is decided on the host, in front of the first launch, so no GPU is needed."""
import ctypes

import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding

OK, EINVAL, ESHAPE, ERANGE = 0, -1, -2, -3
A = 0x100000            # an address that nothing dereferences: all checks come first


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def pages(**kw):
    base = dict(k_dev=A, v_dev=2 * A, page_stride=2 * 16 * 128, head_stride=16 * 128, pos_stride=128, n_pages=10, page_size=16, n_kv_heads=2, head_dim=128, kv_dtype=1)
    base.update(kw)
    return binding.PagesStruct(*[base[f] for f, _ in binding.PagesStruct._fields_])


BAD_PAGES = [(dict(k_dev=None), EINVAL), (dict(v_dev=None), EINVAL), (dict(k_dev=A + 8), EINVAL), (dict(v_dev=A + 2), EINVAL), (dict(kv_dtype=2), EINVAL),
             (dict(head_dim=80), ESHAPE), (dict(head_dim=256), ESHAPE), (dict(n_kv_heads=0), ESHAPE), (dict(page_size=4), ESHAPE), (dict(page_size=24), ESHAPE),
             (dict(page_size=2048), ESHAPE), (dict(n_pages=0), ESHAPE), (dict(n_pages=2 ** 27, page_size=16), ESHAPE), (dict(pos_stride=120), EINVAL),
             (dict(pos_stride=129), EINVAL), (dict(head_stride=64), EINVAL), (dict(pos_stride=2 ** 26 + 8), ESHAPE), (dict(head_stride=16 * 128 + 4), EINVAL), (dict(page_stride=-4096), EINVAL)]


def attention(lib, p, **kw):
    a = dict(table=A, width=4, row_start=A, kv_len=A, n=2, q=A, qs=4 * 128, out=2 * A, os=4 * 128, dtype=1, rows=5, heads=4, scale=0.1, most=0, ws=A, wsb=1 << 40)
    a.update(kw)
    return lib.knnssd_paged_attention(ctypes.byref(p) if p is not None else None, a["table"], a["width"], a["row_start"], a["kv_len"], a["n"], a["q"], a["qs"],
                                      a["out"], a["os"], a["dtype"], a["rows"], a["heads"], a["scale"], a["most"], a["ws"], a["wsb"], None)


def store(lib, p, **kw):
    a = dict(qkv=A, dtype=1, qs=8 * 128, rows=5, heads=4, slots=A, positions=A, base=10000.0, q_out=None, qos=0, k_out=None, kos=0)
    a.update(kw)
    return lib.knnssd_paged_store(ctypes.byref(p) if p is not None else None, *[a[k] for k in ("qkv", "dtype", "qs", "rows", "heads", "slots", "positions", "base", "q_out", "qos", "k_out", "kos")], None)


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_pages(lib, kw, code):
    p = pages(**kw)
    assert attention(lib, p) == code
    assert store(lib, p) == code
    assert lib.knnssd_paged_attention_bytes(ctypes.byref(p), 4, 1) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), EINVAL), (dict(row_start=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(ws=None), EINVAL),
    (dict(ws=A + 16), EINVAL), (dict(wsb=0), EINVAL), (dict(q=A + 8), EINVAL), (dict(out=A + 4), EINVAL), (dict(qs=4 * 128 - 8), EINVAL), (dict(os=4 * 128 + 4), EINVAL),
    (dict(qs=-1024), EINVAL), (dict(dtype=3), EINVAL), (dict(n=0), ERANGE), (dict(n=4097), ERANGE), (dict(rows=0), ERANGE), (dict(width=0), ERANGE), (dict(most=-1), ERANGE),
    (dict(scale=float("nan")), ERANGE), (dict(scale=float("inf")), ERANGE), (dict(heads=3), ESHAPE), (dict(heads=0), ESHAPE),
    (dict(rows=2 ** 23 + 1), ERANGE), (dict(n=4096, heads=4096, qs=4096 * 128, os=4096 * 128), ERANGE)])
def test_paged_attention(lib, kw, code):
    assert attention(lib, pages(), **kw) == code


def test_types_that_do_not_go_together(lib):
    p = pages(kv_dtype=0)
    assert attention(lib, p, dtype=1) == EINVAL
    assert store(lib, p, dtype=1) == EINVAL
    assert lib.knnssd_paged_attention_bytes(ctypes.byref(p), 4, 1) == 0
    assert lib.knnssd_paged_attention_bytes(ctypes.byref(p), 4, 0) > 0
    assert lib.knnssd_paged_attention_bytes(ctypes.byref(pages()), 4, 0) > 0
    assert lib.knnssd_paged_attention_bytes(ctypes.byref(pages()), 3, 1) == 0
    assert lib.knnssd_paged_attention_bytes(None, 4, 1) == 0
    assert attention(lib, None) == EINVAL and store(lib, None) == EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(qkv=None), EINVAL), (dict(slots=None), EINVAL), (dict(positions=None), EINVAL), (dict(qkv=A + 8), EINVAL), (dict(dtype=2), EINVAL), (dict(qs=7 * 128), EINVAL),
    (dict(rows=0), ERANGE), (dict(rows=2 ** 23 + 1), ERANGE), (dict(heads=-1), ERANGE), (dict(base=0.0), ERANGE), (dict(base=float("inf")), ERANGE), (dict(base=float("nan")), ERANGE),
    (dict(q_out=A + 2, qos=512), EINVAL), (dict(q_out=A, qos=511), EINVAL), (dict(k_out=A, kos=128), EINVAL)])
def test_store(lib, kw, code):
    assert store(lib, pages(), **kw) == code


def test_plan(lib):
    def plan(t=None, r=None, cached=A, added=A):
        tables = dict(block_table_dev=A, held_dev=A, free_pages_dev=A, n_free_dev=A, n_requests=3, table_width=4, n_pages=20, page_size=16)
        tables.update(t or {})
        rows = dict(row_start_dev=A, kv_len_dev=A, slots_dev=A, positions_dev=A, result_dev=A, max_rows=9)
        rows.update(r or {})
        ts = binding.PageTablesStruct(*[tables[f] for f, _ in binding.PageTablesStruct._fields_])
        rs = binding.BatchRowsStruct(*[rows[f] for f, _ in binding.BatchRowsStruct._fields_])
        return lib.knnssd_page_plan(ctypes.byref(ts), cached, added, ctypes.byref(rs), None)

    for f in ("block_table_dev", "held_dev", "free_pages_dev", "n_free_dev"):
        assert plan({f: None}) == EINVAL
    for f in ("row_start_dev", "kv_len_dev", "slots_dev", "positions_dev", "result_dev"):
        assert plan(None, {f: None}) == EINVAL
    assert plan(cached=None) == EINVAL and plan(added=None) == EINVAL
    assert plan(dict(n_requests=0)) == ERANGE and plan(dict(n_requests=4097)) == ERANGE and plan(None, dict(max_rows=0)) == ERANGE
    assert plan(dict(page_size=12)) == ESHAPE and plan(dict(n_pages=0)) == ESHAPE and plan(dict(n_pages=2 ** 27)) == ESHAPE
    assert plan(dict(table_width=0)) == ESHAPE and plan(dict(table_width=2 ** 30)) == ESHAPE
    assert lib.knnssd_page_plan(None, A, A, None, None) == EINVAL


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL), (dict(row_start=None), EINVAL), (dict(dtype=5), EINVAL),
    (dict(k=A + 2), EINVAL), (dict(v=A + 2), EINVAL), (dict(ks=128), EINVAL), (dict(vs=2 * 128 + 1), EINVAL), (dict(os=0), EINVAL), (dict(n=0), ERANGE), (dict(n=5000), ERANGE),
    (dict(rows=0), ERANGE), (dict(scale=float("inf")), ERANGE), (dict(dim=96), ESHAPE), (dict(kv_heads=0), ESHAPE), (dict(kv_heads=3), ESHAPE)])
def test_prompt_attention(lib, kw, code):
    a = dict(q=A, qs=512, k=A, ks=256, v=A, vs=256, out=A, os=512, dtype=1, row_start=A, n=2, rows=7, heads=4, kv_heads=2, dim=128, scale=0.1)
    a.update(kw)
    assert lib.knnssd_prompt_attention(*[a[k] for k in ("q", "qs", "k", "ks", "v", "vs", "out", "os", "dtype", "row_start", "n", "rows", "heads", "kv_heads", "dim", "scale")], None) == code


def test_context_pages(lib):
    p = binding.PagesStruct()
    assert lib.knnssd_context_pages(None, 0, 16, ctypes.byref(p)) == EINVAL


def test_the_binding_refuses_tensors_of_other_places_and_shapes():
    t = torch.zeros(4, 2, 16, 64)
    with pytest.raises(ValueError, match="on one GPU"):
        binding.Pages(t, t)
    with pytest.raises(ValueError, match="on a GPU"):
        binding.PageTables(torch.zeros(2, 3, dtype=torch.int32), t, t, t, 16)
    with pytest.raises(ValueError, match="on a GPU"):
        binding.knnssd_prompt_attention(t[0], t[0], t[0], torch.zeros(2, dtype=torch.int32))


def test_the_plain_form_of_the_plan_gives_back_what_it_took():
    """The lists that the GPU's plans are held to: rounds that are undone leave the stack as it was, pages never have two owners."""
    s = B.Stack(4, 8, 25, 8)
    s.plan([0] * 4, [9, 1, 30, 0], 100)
    stack = list(s.free)
    s.plan([9, 1, 30, 0], [20, 9, 3, 1], 100)
    owned = [p for r in range(4) for p in s.table[r][:s.held[r]]]
    assert len(set(owned + s.free)) == 25 == len(owned + s.free)
    s.plan([9, 1, 30, 0], [0] * 4, 1)
    assert s.free == stack
    assert s.plan([0] * 4, [64, 64, 64, 64], 300)["result"] == [0, 0, 4, 0] and s.free == stack
