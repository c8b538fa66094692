"""Batches of requests over a paged cache, as a list of timed cases.

A decoder that serves several requests at once keeps their keys and values in pages of a common pool. One step of it takes,
per request, the positions that are cached already and the rows (tokens) that are new: a prompt, a chunk of one, one token, or
the tokens of a draft that are verified together. Kinds of cases, each one call (page_plan: two) of such a step:

  plan    knnssd_page_plan: pages taken and given back, block tables, slots and positions from the requests' lengths.
          One pass is a round: the pages of the rows that are tried, then the rollback to those that were kept.
  store   knnssd_paged_store: rotary embedding of the queries and keys, keys and values into their slots
  paged   knnssd_paged_attention: the new rows' queries over the pages
  prompt  knnssd_prompt_attention: whole prompts, packed one behind the other, each over itself

Widths are those of the configurations this repository ships (synth.workload: 4/4 heads of 64 in fp32, 32/32, 40/40 and 40/8
heads of 128) or generic ones. Nothing here is tied to a model's values: queries and keys are normal, as projections of a
normed residual stream are.
"""
import math
import random

import torch

own = False

ROPE_BASE = 10000.0
_DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a round of a serving loop: 48 requests in mid-life, one to nine rows each, some of them kept
        dict(name="plan_round_48", kind="plan", requests=48, cached_lo=60, cached_hi=4000, rows_lo=1, rows_hi=9, page=64, pad=0, seed0=1),
        # a full batch of prompts is admitted (about 100 000 rows), later all of its pages go back
        dict(name="plan_admit_256", kind="plan", requests=256, cached_lo=0, cached_hi=0, rows_lo=16, rows_hi=1500, page=16, pad=37, seed0=2),
        # the smallest: three requests of the fp32 configuration, one to five rows
        dict(name="store_tiny_fp32", kind="store", requests=3, cached_lo=5, cached_hi=60, rows_lo=1, rows_hi=5, page=16, pad=0, heads=4, kv_heads=4,
             dim=64, q="fp32", kv="fp32", order="head", seed0=3),
        # prompts of a 40-head model
        dict(name="store_prompts_13b", kind="store", requests=6, cached_lo=0, cached_hi=0, rows_lo=900, rows_hi=2100, page=64, pad=100, heads=40, kv_heads=40,
             dim=128, q="bf16", kv="bf16", order="head", seed0=4),
        # one request, one token: what latency is left
        dict(name="paged_1row_qwen", kind="paged", requests=1, cached_lo=1500, cached_hi=1500, rows_lo=1, rows_hi=1, page=64, pad=0, heads=40, kv_heads=8,
             dim=128, q="bf16", kv="bf16", order="head", seed0=5),
        # verified drafts of a batch, grouped heads, ordinary contexts
        dict(name="paged_verify_qwen", kind="paged", requests=32, cached_lo=200, cached_hi=4000, rows_lo=1, rows_hi=9, page=64, pad=0, heads=40, kv_heads=8,
             dim=128, q="bf16", kv="bf16", order="head", seed0=6),
        # the same with queries in 32 bits, as this library's own passes keep them, a head of keys for each head of queries
        dict(name="paged_verify_13b_fp32q", kind="paged", requests=12, cached_lo=300, cached_hi=3500, rows_lo=2, rows_hi=5, page=32, pad=3, heads=40, kv_heads=40,
             dim=128, q="fp32", kv="bf16", order="head", seed0=7),
        # two requests far into long documents: few rows, a long axis
        dict(name="paged_long_qwen", kind="paged", requests=2, cached_lo=90000, cached_hi=110000, rows_lo=4, rows_hi=6, page=128, pad=0, heads=40, kv_heads=8,
             dim=128, q="bf16", kv="bf16", order="position", seed0=8),
        # chunks of long prompts beside single rows of others
        dict(name="paged_chunks_qwen", kind="paged", requests=8, cached_lo=700, cached_hi=9000, rows_lo=1, rows_hi=900, page=64, pad=11, heads=40, kv_heads=8,
             dim=128, q="bf16", kv="bf16", order="head", seed0=9),
        # prompts of the fp32 configuration
        dict(name="prompt_tiny_fp32", kind="prompt", requests=3, rows_lo=1, rows_hi=45, pad=0, heads=4, kv_heads=4, dim=64, q="fp32", seed0=10),
        # few-shot prompts of odd lengths, heads of 64
        dict(name="prompt_ragged_64", kind="prompt", requests=9, rows_lo=40, rows_hi=1700, pad=50, heads=32, kv_heads=8, dim=64, q="bf16", seed0=11),
        # two prompts of the length that the task-stream configuration uses
        dict(name="prompt_13b_4096", kind="prompt", requests=2, rows_lo=4000, rows_hi=4200, pad=0, heads=40, kv_heads=40, dim=128, q="bf16", seed0=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "store", "paged", "paged", "paged", "prompt", "prompt"])
    c = dict(kind=kind, seed0=rng.randrange(1 << 20))
    if kind == "plan":
        c["requests"] = _log_int(rng, 1, 700)
        fresh = rng.random() < 0.4
        c["cached_lo"] = 0 if fresh else _log_int(rng, 1, 300)
        c["cached_hi"] = 0 if fresh else c["cached_lo"] + _log_int(rng, 1, 4000)
        c["rows_lo"] = rng.choice([0, 1, 1, 16])
        c["rows_hi"] = max(c["rows_lo"], _log_int(rng, 1, 16) if not fresh else _log_int(rng, 16, 100000 // c["requests"] + 20))
        c["page"] = rng.choice([8, 16, 32, 64, 128, 256])
        c["pad"] = rng.choice([0, 0, _log_int(rng, 1, 500)])
        return c
    kv_heads = rng.choice([1, 2, 4, 8, 8, 20, 40])
    groups = rng.choice([1, 1, 2, 4, 5, 8]) if kv_heads <= 8 else rng.choice([1, 2])
    c.update(heads=kv_heads * groups, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]))
    c["q"], c["kv"] = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
    if kind == "prompt":
        c.pop("kv")
        c["requests"] = rng.randint(1, 12)
        c["rows_lo"] = rng.choice([0, 1, 16, 100])
        most = 2500 if c["q"] == "bf16" else 600
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 1, most * 2 // (1 + c["requests"]))
        c["pad"] = rng.choice([0, 0, _log_int(rng, 1, 200)])
        return c
    c["page"] = rng.choice([16, 32, 64, 64, 128, 256])
    c["order"] = rng.choice(["head", "head", "position"])
    c["pad"] = rng.choice([0, 0, rng.randint(1, 60)])
    if kind == "store":
        c["requests"] = _log_int(rng, 1, 60)
        c["cached_lo"] = rng.choice([0, 0, 5])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 1, 4000)
        c["rows_lo"] = rng.choice([0, 1])
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 1, 1 + 6000 // c["requests"])
        return c
    form = rng.choice(["round", "round", "long", "chunk"])
    c["rows_lo"] = rng.choice([0, 1, 1])
    if form == "round":
        c["requests"] = _log_int(rng, 1, 64)
        c["cached_lo"] = rng.choice([0, 1, 100])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 10, 3000)
        c["rows_hi"] = c["rows_lo"] + rng.randint(1, 15)
    elif form == "long":
        c["requests"] = rng.randint(1, 3)
        c["cached_lo"] = _log_int(rng, 3000, 40000)
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 1, 20000)
        c["rows_hi"] = c["rows_lo"] + rng.randint(1, 8)
    else:
        c["requests"] = rng.randint(1, 8)
        c["cached_lo"] = rng.choice([0, 300])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 10, 4000 if c["q"] == "bf16" else 1000)
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 17, 800 if c["q"] == "bf16" else 150)
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _lengths(case, seed=0):
    """Per request: rows, cached positions, rows that are kept. The sizes are the case's (work() knows them); which request has which is the seed's."""
    r = random.Random(case["seed0"])
    rows = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["requests"])]
    if not any(rows):
        rows[0] = 1
    lo, hi = case.get("cached_lo", 0), case.get("cached_hi", 0)
    cached = [r.randint(lo, hi) for _ in rows]
    both = list(zip(rows, cached))
    random.Random(seed).shuffle(both)
    rows, cached = [a for a, _ in both], [b for _, b in both]
    kept = [0 if not hi else r.randint(min(1, a), a) for a in rows]
    return rows, cached, kept


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed * 1000003 + case["seed0"])
    rows, cached, kept = _lengths(case, seed)
    n, total = case["requests"], sum(rows)
    s = dict(case=case, total=total, most_rows=max(rows), cap=total + case["pad"])
    start = [0]
    for a in rows:
        start.append(start[-1] + a)
    s["row_start"] = _int32(start)
    if own:
        from paper_2505_16162_amd import binding
    if case["kind"] == "prompt":
        q, heads, kv_heads, dim = _DT[case["q"]], case["heads"], case["kv_heads"], case["dim"]
        s["longest"] = max(rows)
        s["qkv"] = _normal(gen, (s["cap"], (heads + 2 * kv_heads) * dim), q)     # queries | keys | values of a row, as one product gives them
        s["out"] = torch.zeros((s["cap"], heads, dim), dtype=q, device="cuda")
        return s
    page = case["page"]
    lens = [a + b for a, b in zip(rows, cached)]
    s["longest"] = max(lens)
    pages_of = lambda v: -(-v // page)  # noqa: E731
    width = max(pages_of(v) for v in lens) + 1
    need = sum(pages_of(v) for v in lens)
    n_pages = need + max(2, need // 8)
    ids = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)     # pages have been through many hands
    held = [pages_of(v) for v in (cached if case["kind"] == "plan" else lens)]
    column = torch.arange(width, device="cuda")
    h = torch.tensor(held, device="cuda")
    first = torch.cumsum(h, 0) - h
    s["block_table"] = torch.where(column[None] < h[:, None], ids[(first[:, None] + column[None]).clamp(max=n_pages - 1)], -1).to(torch.int32)
    s["width"], s["n_pages"] = width, n_pages
    if case["kind"] == "plan":
        used = sum(held)
        s["held"] = _int32(held)
        s["free_pages"] = torch.cat([ids[used:], torch.full((used,), -1, dtype=torch.int32, device="cuda")])
        s["n_free"] = _int32([n_pages - used])
        s["cached"], s["added"] = _int32(cached), _int32(rows)
        s["kept"] = _int32([b + c for b, c in zip(cached, kept)])
        s["none"] = _int32([0] * n)
        s["tables"] = binding.PageTables(s["block_table"], s["held"], s["free_pages"], s["n_free"], page) if own else None
        s["rows"] = (binding.BatchRows(n, s["cap"]), binding.BatchRows(n, 1)) if own else None
        return s
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    s["kv_len"] = _int32(lens)
    if case["order"] == "head":
        shape, turn = (n_pages, kv_heads, page, dim), (0, 1, 2, 3)
    else:
        shape, turn = (n_pages, page, kv_heads, dim), (0, 2, 1, 3)
    s["k"] = _normal(gen, shape, _DT[case["kv"]]).permute(turn)         # [page][kv head][position][dim], however it lies in memory
    s["v"] = _normal(gen, shape, _DT[case["kv"]]).permute(turn)
    s["pages"] = binding.Pages(s["k"], s["v"]) if own else None
    if case["kind"] == "store":
        t = torch.arange(s["cap"], device="cuda")
        request = torch.searchsorted(s["row_start"][1:].contiguous(), t, right=True).clamp(max=n - 1)
        pos = t - s["row_start"][request] + _int32(cached)[request]
        at = s["block_table"][request, (pos // page).clamp(max=width - 1)] * page + pos % page
        live = t < total
        s["positions"] = torch.where(live, pos, -1).to(torch.int32)
        s["slots"] = torch.where(live, at, -1).to(torch.int32)
        s["qkv"] = _normal(gen, (s["cap"], (heads + 2 * kv_heads) * dim), _DT[case["q"]])
        s["q_out"] = torch.zeros((s["cap"], heads, dim), dtype=_DT[case["q"]], device="cuda")
        return s
    s["q"] = _normal(gen, (s["cap"], heads, dim), _DT[case["q"]])
    s["out"] = torch.zeros((s["cap"], heads, dim), dtype=_DT[case["q"]], device="cuda")
    s["workspace"] = binding.paged_attention_workspace(s["pages"], heads, _DT[case["q"]]) if own else None
    return s


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plan(s, cached, added, cap):
    """Pages are a stack: what goes back is pushed in descending order of request and page, what is needed is popped in ascending order."""
    page, width, table, held = s["case"]["page"], s["width"], s["block_table"], s["held"]
    length = cached + added
    need = (length + page - 1) // page
    back, take = (held - need).clamp(min=0), (need - held).clamp(min=0)
    n_back, n_take, n_free = back.sum(), take.sum(), s["n_free"][0]
    column = torch.arange(width, device=table.device)[None]
    goes = (column >= need[:, None]) & (column < held[:, None])
    comes = (column >= held[:, None]) & (column < need[:, None])
    rank_back = (torch.cumsum(back, 0) - back)[:, None] + column - need[:, None]
    rank_take = (torch.cumsum(take, 0) - take)[:, None] + column - held[:, None]
    spare = torch.full((table.numel() + 1,), -1, dtype=torch.int32, device=table.device)       # the pages that go back, ascending; the last entry is a bin
    spare[torch.where(goes, rank_back, table.numel()).reshape(-1)] = table.reshape(-1)
    pool = s["free_pages"]
    from_pool = (n_free - 1 - (rank_take - n_back)).clamp(0, pool.numel() - 1)
    fresh = torch.where(rank_take < n_back, spare[rank_take.clamp(0, table.numel())], pool[from_pool])
    new_table = torch.where(comes, fresh, torch.where(goes, -1, table)).to(torch.int32)
    left = n_free + n_back - n_take
    i = torch.arange(pool.numel(), device=table.device)
    pushed = spare[(n_back - 1 - (i - n_free)).clamp(0, table.numel())]
    new_pool = torch.where(i >= left, -1, torch.where(i >= n_free, pushed, pool)).to(torch.int32)
    start = torch.cat([torch.zeros_like(added[:1]), torch.cumsum(added, 0).to(torch.int32)])
    t = torch.arange(cap, device=table.device)
    request = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=held.numel() - 1)
    pos = t - start[request] + cached[request]
    slot = new_table[request, (pos // page).clamp(max=width - 1)] * page + pos % page
    live = t < start[-1]
    s["block_table"].copy_(new_table)
    s["held"].copy_(need)
    s["free_pages"].copy_(new_pool)
    s["n_free"].copy_(left[None])
    result = torch.stack([start[-1], n_take - n_back, torch.zeros_like(n_take), length.max()]).to(torch.int32)
    return dict(row_start=start, kv_len=length, slots=torch.where(live, slot, -1).to(torch.int32), positions=torch.where(live, pos, -1).to(torch.int32), result=result)


def _rotate(x, positions):
    """Pairs (i, i + dim/2) of each head turned by position * base^(-2i/dim); angles in 64 bits, products in 32."""
    half = x.shape[-1] // 2
    turn = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device=x.device) * 2 / x.shape[-1])
    angle = positions.double()[:, None, None] * turn
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _store(s):
    heads, kv_heads, dim, page = (s["case"][k] for k in ("heads", "kv_heads", "dim", "page"))
    rows = s["qkv"].shape[0]
    x = s["qkv"].float().view(rows, heads + 2 * kv_heads, dim)
    live = s["slots"] >= 0
    turned = _rotate(x[:, :heads + kv_heads], s["positions"])
    s["q_out"].copy_(torch.where(live[:, None, None], turned[:, :heads].to(s["q_out"].dtype), s["q_out"]))
    # a row that goes nowhere repeats the first live row's write
    src = torch.where(live, torch.arange(rows, device=x.device), live.int().argmax())
    at, keys, values = s["slots"][src].long(), turned[src, heads:], x[src, heads + kv_heads:]
    s["k"][at // page, :, at % page] = keys.to(s["k"].dtype)
    s["v"][at // page, :, at % page] = values.to(s["v"].dtype)
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _attend(q, k, v, cached, rows, groups, dtype):
    """q [requests][rows][heads][dim], k and v [requests][kv head][positions][dim], all in 32 bits: softmax over the positions up to a row's own."""
    n, m, heads, dim = q.shape
    kv_heads, length = k.shape[1], k.shape[2]
    q = q.view(n, m, kv_heads, groups, dim).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, m * groups, dim) * dim ** -0.5
    score = (q @ k.transpose(-1, -2).contiguous()).view(n, kv_heads, m, groups, length)
    at = torch.arange(length, device=q.device)
    own_at = cached[:, None] + torch.arange(m, device=q.device)[None]
    hidden = (at[None, None] > own_at[:, :, None])[:, None, :, None]
    score = score.masked_fill_(hidden, -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    p = score.div_(score.sum(-1, keepdim=True)).view(n, kv_heads, m * groups, length)
    return (p @ v).view(n, kv_heads, m, groups, dim).permute(0, 2, 1, 3, 4).reshape(n, m, heads, dim).to(dtype)


def _padded(s):
    """Row of the packed batch for each (request, row), and whether there is one."""
    start = s["row_start"].long()
    i = torch.arange(s["most_rows"], device=start.device)[None]
    return (start[:-1, None] + i).clamp(max=s["cap"] - 1), i < (start[1:] - start[:-1])[:, None]


def _packed(s, padded):
    """The packed batch back from (request, row); rows behind the last request stay as they were."""
    start = s["row_start"].long()
    t = torch.arange(s["cap"], device=start.device)
    request = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=start.numel() - 2)
    rows = padded[request, (t - start[request]).clamp(max=s["most_rows"] - 1)]
    s["out"].copy_(torch.where((t < start[-1])[:, None, None], rows, s["out"]))
    return s["out"]


def _paged(s):
    heads, kv_heads, dim, page = (s["case"][k] for k in ("heads", "kv_heads", "dim", "page"))
    row, _ = _padded(s)
    used = -(-s["longest"] // page)
    table = s["block_table"][:, :used].clamp(min=0).long()
    n = table.shape[0]
    k = s["k"][table].float().permute(0, 2, 1, 3, 4).reshape(n, kv_heads, used * page, dim)
    v = s["v"][table].float().permute(0, 2, 1, 3, 4).reshape(n, kv_heads, used * page, dim)
    cached = s["kv_len"] - (s["row_start"][1:] - s["row_start"][:-1])
    return _packed(s, _attend(s["q"].float()[row], k, v, cached, row, heads // kv_heads, s["q"].dtype))


def _prompt(s):
    heads, kv_heads, dim = (s["case"][k] for k in ("heads", "kv_heads", "dim"))
    row, live = _padded(s)
    x = s["qkv"].float()[row].view(row.shape[0], row.shape[1], heads + 2 * kv_heads, dim)
    k = x[:, :, heads:heads + kv_heads].permute(0, 2, 1, 3).contiguous()
    v = x[:, :, heads + kv_heads:].permute(0, 2, 1, 3).contiguous()
    return _packed(s, _attend(x[:, :, :heads].contiguous(), k, v, torch.zeros_like(s["row_start"][1:]), row, heads // kv_heads, s["qkv"].dtype))


# ---------------------------------------------------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------------------------------------------------
def _own(s, kind):
    from paper_2505_16162_amd import binding
    if kind == "plan":
        binding.knnssd_page_plan(s["tables"], s["rows"][0], s["cached"], s["added"])
        binding.knnssd_page_plan(s["tables"], s["rows"][1], s["kept"], s["none"])
        r = s["rows"][0]
        return dict(row_start=r.row_start, kv_len=r.kv_len, slots=r.slots, positions=r.positions, result=r.result, table=s["block_table"], held=s["held"],
                    free=s["free_pages"], n_free=s["n_free"], back=s["rows"][1].result)
    if kind == "store":
        binding.knnssd_paged_store(s["pages"], s["qkv"], s["slots"], s["positions"], rope_base=ROPE_BASE, q_out=s["q_out"])
        return dict(q=s["q_out"], k=s["k"], v=s["v"])
    if kind == "paged":
        return binding.knnssd_paged_attention(s["pages"], s["block_table"], s["row_start"], s["kv_len"], s["q"], s["workspace"], out=s["out"],
                                              most_rows=s["most_rows"])
    c = s["case"]
    x = s["qkv"].view(s["cap"], c["heads"] + 2 * c["kv_heads"], c["dim"])
    q, k, v = x.split([c["heads"], c["kv_heads"], c["kv_heads"]], 1)
    return binding.knnssd_prompt_attention(q, k, v, s["row_start"], out=s["out"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    if kind == "plan":
        r = _plan(s, s["cached"], s["added"], s["cap"])
        back = _plan(s, s["kept"], s["none"], 1)
        return dict(r, table=s["block_table"], held=s["held"], free=s["free_pages"], n_free=s["n_free"], back=back["result"])
    return {"store": _store, "paged": _paged, "prompt": _prompt}[kind](s)


def work(case):
    rows, cached, kept = _lengths(case)
    total = sum(rows)
    if case["kind"] == "plan":
        pages = [-(-(a + b) // case["page"]) for a, b in zip(rows, cached)]
        back = [p - -(-(b + c) // case["page"]) for p, b, c in zip(pages, cached, kept)]
        # lengths and pages held in, starts, lengths, a slot and a position a row out; a page changes hands: read once, written once
        return dict(bytes=4 * (2 * 6 * len(rows) + 2 * (total + case["pad"]) + 4 * sum(back)), flops=0)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    qb = 4 if case["q"] == "fp32" else 2
    kvb = qb if case["kind"] == "prompt" else 4 if case["kv"] == "fp32" else 2
    if case["kind"] == "store":
        return dict(bytes=total * dim * (qb * (2 * heads + 2 * kv_heads) + kvb * 2 * kv_heads) + 8 * total, flops=3 * total * dim * (heads + kv_heads))
    seen = sum(a * b + a * (a + 1) // 2 for a, b in zip(rows, cached))       # (row, position) pairs
    lens = sum(a + b for a, b in zip(rows, cached) if a)
    return dict(bytes=2 * total * heads * dim * qb + 2 * lens * kv_heads * dim * kvb, flops=4 * seen * heads * dim)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_plan(s):
    """A stack of pages and lists, request by request."""
    page = s["case"]["page"]
    table = s["block_table"].tolist()
    held = s["held"].tolist()
    stack = s["free_pages"].tolist()[:s["n_free"].item()]

    def step(cached, added, cap):
        lens = [a + b for a, b in zip(cached, added)]
        need = [-(-v // page) for v in lens]
        before = len(stack)
        for r in reversed(range(len(lens))):
            while held[r] > need[r]:
                held[r] -= 1
                stack.append(table[r][held[r]])
                table[r][held[r]] = -1
        for r in range(len(lens)):
            while held[r] < need[r]:
                table[r][held[r]] = stack.pop()
                held[r] += 1
        start, slots, positions = [0], [], []
        for r, (c, a) in enumerate(zip(cached, added)):
            start.append(start[-1] + a)
            positions += range(c, c + a)
            slots += [table[r][p // page] * page + p % page for p in range(c, c + a)]
        fill = [-1] * (cap - len(slots))
        return dict(row_start=start, kv_len=lens, slots=slots + fill, positions=positions + fill, result=[start[-1], before - len(stack), 0, max(lens)])

    got = step(s["cached"].tolist(), s["added"].tolist(), s["cap"])
    back = step(s["kept"].tolist(), s["none"].tolist(), 1)["result"]
    got.update(table=table, held=held, free=stack + [-1] * (s["n_pages"] - len(stack)), n_free=[len(stack)], back=back)
    return {k: _int32(v) for k, v in got.items()}


def _exact_rows(q, k, v, cached):
    """One request in 64 bits, a head of keys at a time: q [rows][heads][dim], k and v [positions][kv heads][dim]."""
    m, heads, dim = q.shape
    groups = heads // k.shape[1]
    hidden = torch.arange(k.shape[0], device=q.device)[None] > cached + torch.arange(m, device=q.device)[:, None]
    out = torch.empty((m, heads, dim), dtype=torch.float64, device=q.device)
    for h in range(heads):
        score = q[:, h].double() @ k[:, h // groups].double().t().contiguous() / math.sqrt(dim)
        out[:, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[:, h // groups].double()
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return _exact_plan(s)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "store":
        x = s["qkv"].double().view(-1, heads + 2 * kv_heads, dim)
        half = dim // 2
        place = torch.polar(torch.ones(()).double().cuda(), s["positions"].double()[:, None] * torch.exp(torch.arange(half, device="cuda").double() * (-2 / dim * math.log(ROPE_BASE))))
        turned = torch.complex(x[..., :half], x[..., half:]) * place[:, None]
        turned = torch.cat([turned.real, turned.imag], -1)
        out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
        live = (s["slots"] >= 0).nonzero()[:, 0]
        at = s["slots"][live].long()
        out[live] = turned[live, :heads]
        k[at // case["page"], :, at % case["page"]] = turned[live, heads:heads + kv_heads]
        v[at // case["page"], :, at % case["page"]] = x[live, heads + kv_heads:]
        return dict(q=out, k=k, v=v)
    out = s["out"].double()
    start = s["row_start"].tolist()
    for r, (a, b) in enumerate(zip(start, start[1:])):
        if a == b:
            continue
        if case["kind"] == "prompt":
            x = s["qkv"][a:b].view(b - a, heads + 2 * kv_heads, dim)
            q, k, v = x.split([heads, kv_heads, kv_heads], 1)
        else:
            length = s["kv_len"][r].item()
            at = torch.arange(length, device="cuda")
            pages = s["block_table"][r, at // case["page"]].long()
            q, k, v = s["q"][a:b], s["k"][pages, :, at % case["page"]], s["v"][pages, :, at % case["page"]]
        out[a:b] = _exact_rows(q, k, v, k.shape[0] - (b - a))
    return out
