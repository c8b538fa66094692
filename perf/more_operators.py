"""Rounds of a batch with trees of drafted tokens, as a list of timed cases.

A decoder that drafts several candidates for a position has, per request, a tree of new rows: row 0 is the last token that is certain, every
other row is a drafted token whose parent is an earlier row. All rows go through the model together, each seeing the cache and its own ancestors.
Then the drafts are tried against the model's probabilities, from random numbers that the caller brings, and the cache's entries of the
path that was kept are put side by side. Kinds of cases, each one call of such a round:

  plan    knnssd_tree_plan: positions and masks of ancestors from the rows' parents
  tree    knnssd_tree_attention: the rows' queries over the pages, each row over the cached positions and its ancestors
  verify  knnssd_tree_verify: the accepted path and the next token, from logits, drafted tokens and uniform numbers
  keep    knnssd_tree_keep: the kept rows' keys and values to the positions behind the cached ones, in all blocks of a model

Widths are those of the configurations this repository ships (synth.workload: 4/4 heads of 64 in fp32, 32/32, 40/40 and 40/8
heads of 128, vocabularies of 1024, 32000 and 152064) or generic ones.
"""
import math
import random
from collections import Counter

import torch

own = False

_DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # a handful of requests with ordinary trees: what latency is left
        dict(name="plan_8", kind="plan", requests=8, cached_lo=60, cached_hi=4000, rows_lo=4, rows_hi=26, shape="tree", words=1, pad=0, seed0=1),
        # a full batch with very wide trees
        dict(name="plan_192_wide", kind="plan", requests=192, cached_lo=10, cached_hi=4000, rows_lo=20, rows_hi=500, shape="tree", words=8, pad=37, seed0=2),
        # the fp32 configuration: three requests, short contexts
        dict(name="tree_tiny_fp32", kind="tree", requests=3, cached_lo=5, cached_hi=60, rows_lo=3, rows_hi=17, shape="tree", words=1, page=16, pad=0, heads=4,
             kv_heads=4, dim=64, q="fp32", kv="fp32", order="head", seed0=3),
        # one request with one tree, grouped heads
        dict(name="tree_1req_qwen", kind="tree", requests=1, cached_lo=1500, cached_hi=1500, rows_lo=26, rows_hi=26, shape="tree", words=1, page=64, pad=0, heads=40,
             kv_heads=8, dim=128, q="bf16", kv="bf16", order="head", seed0=4),
        # a batch in mid-life, trees of 8 to 64 tokens
        dict(name="tree_batch_qwen", kind="tree", requests=24, cached_lo=200, cached_hi=4000, rows_lo=8, rows_hi=64, shape="tree", words=1, page=64, pad=5, heads=40,
             kv_heads=8, dim=128, q="bf16", kv="bf16", order="head", seed0=5),
        # small trees, queries in 32 bits as this library's own passes keep them, a head of keys for each head of queries
        dict(name="tree_13b_fp32q", kind="tree", requests=10, cached_lo=300, cached_hi=3500, rows_lo=2, rows_hi=16, shape="tree", words=1, page=32, pad=3, heads=40,
             kv_heads=40, dim=128, q="fp32", kv="bf16", order="head", seed0=6),
        # two requests far into long documents
        dict(name="tree_long_qwen", kind="tree", requests=2, cached_lo=90000, cached_hi=110000, rows_lo=60, rows_hi=64, shape="tree", words=1, page=128, pad=0, heads=40,
             kv_heads=8, dim=128, q="bf16", kv="bf16", order="position", seed0=7),
        # one request, the draft's most likely tokens tried in turn
        dict(name="verify_given_1req", kind="verify", requests=1, rows_lo=26, rows_hi=26, shape="tree", pad=0, vocab=32000, gap=0, dtype="bf16", drawn=False, greedy=0.0, seed0=8),
        # a batch of chains of up to eight drawn tokens, the widest vocabulary
        dict(name="verify_chains_qwen", kind="verify", requests=32, rows_lo=1, rows_hi=9, shape="chain", pad=0, vocab=152064, gap=0, dtype="bf16", drawn=True, greedy=0.1, seed0=9),
        # trees of drawn tokens, logits in 32 bits, rows that lie apart
        dict(name="verify_trees_fp32", kind="verify", requests=12, rows_lo=8, rows_hi=48, shape="tree", pad=3, vocab=32000, gap=5, dtype="fp32", drawn=True, greedy=0.0, seed0=10),
        # the fp32 configuration's four blocks
        dict(name="keep_tiny_fp32", kind="keep", requests=3, cached_lo=5, cached_hi=60, rows_lo=5, rows_hi=17, page=16, pad=0, blocks=4, kv_heads=4, dim=64, kv="fp32",
             order="head", seed0=11),
        # all 48 blocks of a model with grouped heads
        dict(name="keep_batch_qwen", kind="keep", requests=32, cached_lo=10, cached_hi=150, rows_lo=8, rows_hi=64, page=16, pad=7, blocks=48, kv_heads=8, dim=128, kv="bf16",
             order="head", seed0=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "tree", "tree", "tree", "verify", "verify", "verify", "keep"])
    c = dict(kind=kind, seed0=rng.randrange(1 << 20))
    c["pad"] = rng.choice([0, 0, _log_int(rng, 1, 60)])
    if kind == "plan":
        c["requests"] = _log_int(rng, 1, 500)
        c["cached_lo"] = rng.choice([0, 1, 60])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 1, 4000)
        c["rows_lo"] = rng.choice([0, 1, 4])
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 1, min(1000, 50000 // c["requests"]))
        c["shape"] = rng.choice(["tree", "tree", "chain", "forest"])
        c["words"] = -(-c["rows_hi"] // 64) + rng.choice([0, 0, 1]) if c["rows_hi"] <= 960 else 16
        return c
    if kind == "verify":
        c["vocab"] = rng.choice([1024, 32000, 152064, _log_int(rng, 2, 160000), _log_int(rng, 500, 160000)])
        c["gap"] = rng.choice([0, 0, 8, rng.randint(1, 300)])
        c["dtype"] = rng.choice(["bf16", "fp32"])
        c["drawn"] = rng.random() < 0.6
        c["greedy"] = rng.choice([0.0, 0.0, 0.3, 1.0])
        c["shape"] = rng.choice(["chain", "tree"])
        c["requests"] = _log_int(rng, 1, 48)
        c["rows_lo"] = rng.choice([1, 1, 2])
        most = max(2, min(64, 24000000 // (c["requests"] * c["vocab"])))
        c["rows_hi"] = c["rows_lo"] + rng.randint(0, min(most, 12) if c["shape"] == "chain" else most)
        return c
    c["page"] = rng.choice([8, 16, 32, 64, 64, 128, 256])
    c["order"] = rng.choice(["head", "head", "position"])
    if kind == "keep":
        c["requests"] = _log_int(rng, 1, 40)
        c["cached_lo"] = rng.choice([0, 5])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 1, 200)
        c["rows_lo"] = rng.choice([1, 4])
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 1, 80)
        c["kv"] = rng.choice(["bf16", "bf16", "fp32"])
        c["kv_heads"] = rng.choice([1, 2, 4, 8])
        c["dim"] = rng.choice([64, 128])
        position = 2 * c["kv_heads"] * c["dim"] * (4 if c["kv"] == "fp32" else 2)
        c["blocks"] = _log_int(rng, 1, max(1, min(60, 700000000 // (position * c["requests"] * (c["cached_hi"] + c["rows_hi"])))))
        return c
    kv_heads = rng.choice([1, 2, 4, 8, 8, 20, 40])
    groups = rng.choice([1, 1, 2, 4, 5, 8]) if kv_heads <= 8 else rng.choice([1, 2])
    c.update(heads=kv_heads * groups, kv_heads=kv_heads, dim=rng.choice([64, 128, 128]))
    c["q"], c["kv"] = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
    c["shape"] = rng.choice(["tree", "tree", "tree", "forest", "chain"])
    c["rows_lo"] = rng.choice([0, 1, 4])
    form = rng.choice(["round", "round", "long", "wide"])
    if form == "round":
        c["requests"] = _log_int(rng, 1, 32)
        c["cached_lo"] = rng.choice([0, 1, 100])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 10, 3000)
        c["rows_hi"] = c["rows_lo"] + rng.randint(1, 60)
    elif form == "long":
        c["requests"] = rng.randint(1, 3)
        c["cached_lo"] = _log_int(rng, 3000, 40000)
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 1, 20000)
        c["rows_hi"] = c["rows_lo"] + rng.randint(1, 40)
    else:
        c["requests"] = rng.randint(1, 6)
        c["cached_lo"] = rng.choice([0, 300])
        c["cached_hi"] = c["cached_lo"] + _log_int(rng, 10, 3000 if c["q"] == "bf16" else 1000)
        c["rows_hi"] = c["rows_lo"] + _log_int(rng, 60, 300 if c["q"] == "bf16" else 150)
    c["words"] = -(-c["rows_hi"] // 64)
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _parents(r, n, shape):
    """Parents of n rows: a chain, a tree in which a node has a few children, or several such trees."""
    if shape == "chain":
        return list(range(-1, n - 1))
    got = [-1] * min(n, 1)
    for i in range(1, n):
        got.append(-1 if shape == "forest" and r.random() < 0.2 else r.randint((i - 1) // 3, max((i - 1) // 3, (i - 1) // 2 + 1 if i > 2 else 0)))
    return [min(p, i - 1) for i, p in enumerate(got)]


def _path(r, parents):
    """A way from the root towards a leaf on which no entry goes where another one comes from, so that a second pass over the moved
    cache finds what the first one found."""
    for _ in range(50):
        path = [0]
        while True:
            children = [i for i, p in enumerate(parents) if p == path[-1] and i]
            if not children or r.random() < 0.15:
                break
            path.append(r.choice(children))
        if not {j for j, i in enumerate(path) if i != j} & {i for j, i in enumerate(path) if i != j}:
            return path
    return [0]


def _structure(case, seed=0):
    """Per request: parents, cached positions, a kept path. The sizes are the case's (work() knows them); which request has which is the seed's."""
    r = random.Random(case["seed0"])
    got = []
    for i in range(case["requests"]):
        n = r.randint(case["rows_lo"], case["rows_hi"])
        if i == 0:
            n = max(n, 1)
        parents = _parents(r, n, case.get("shape", "tree"))
        got.append((parents, r.randint(case.get("cached_lo", 0), case.get("cached_hi", 0)), _path(r, parents) if case["kind"] == "keep" else []))
    random.Random(seed).shuffle(got)
    return [g[0] for g in got], [g[1] for g in got], [g[2] for g in got]


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _uniform(gen, n):
    return torch.rand(n, generator=gen, device="cuda")


def _bits(parents, words):
    """Masks of ancestors as rows of `words` 64-bit words, on the host."""
    got = []
    for i, p in enumerate(parents):
        got.append((got[p] if p >= 0 else 0) | 1 << i)
    out = [[(m >> 64 * w) & (2 ** 64 - 1) for w in range(words)] for m in got]
    return [[v - 2 ** 64 if v >= 2 ** 63 else v for v in m] for m in out]


def prepare(case, seed):
    gen = torch.Generator("cuda")
    gen.manual_seed(seed * 1000003 + case["seed0"])
    parents, cached, paths = _structure(case, seed)
    rows = [len(p) for p in parents]
    n, total = case["requests"], sum(rows)
    cap = total + case["pad"]
    s = dict(case=case, total=total, most_rows=max(rows), cap=cap)
    start = [0]
    for a in rows:
        start.append(start[-1] + a)
    s["row_start"] = _int32(start)
    flat = [p for ps in parents for p in ps]
    s["parents"] = _int32(flat + [-1] * case["pad"])
    s["most_children"] = max(c for ps in parents for c in Counter(p for p in ps if p >= 0).values() or [0])
    if own:
        from paper_2505_16162_amd import binding
    if case["kind"] == "verify":
        _prepare_verify(s, gen, flat, start)
        if own:
            s["workspace"] = binding.tree_verify_workspace(cap, n, case["vocab"], case["drawn"])
        return s
    lens = [a + b for a, b in zip(rows, cached)]
    s["longest"] = max(lens)
    s["kv_len"] = _int32(lens)
    if case["kind"] == "plan":
        s["positions"] = torch.full((cap,), -1, dtype=torch.int32, device="cuda")
        s["masks"] = torch.zeros((cap, case["words"]), dtype=torch.int64, device="cuda")
        return s
    page = case["page"]
    pages_of = [-(-v // page) for v in lens]
    width, need = max(pages_of) + 1, sum(pages_of)
    n_pages = need + max(2, need // 8)
    ids = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)     # pages have been through many hands
    column = torch.arange(width, device="cuda")
    h = torch.tensor(pages_of, device="cuda")
    first = torch.cumsum(h, 0) - h
    s["block_table"] = torch.where(column[None] < h[:, None], ids[(first[:, None] + column[None]).clamp(max=n_pages - 1)], -1).to(torch.int32)
    kv_heads, dim, blocks = case["kv_heads"], case["dim"], case.get("blocks", 1)
    if case["order"] == "head":
        shape, turn = (blocks, 2, n_pages, kv_heads, page, dim), (0, 1, 2, 3, 4, 5)
    else:
        shape, turn = (blocks, 2, n_pages, page, kv_heads, dim), (0, 1, 2, 4, 3, 5)
    s["cache"] = _normal(gen, shape, _DT[case["kv"]]).permute(turn)      # [block][keys, values][page][kv head][position][dim], however it lies in memory
    if case["kind"] == "keep":
        s["path"] = _int32([v for p, a in zip(paths, rows) for v in p + [-1] * (a - len(p))] + [-1] * case["pad"])
        s["n_path"] = _int32([len(p) for p in paths])
        s["cached"] = torch.zeros(n, dtype=torch.int32, device="cuda")
        s["blocks"] = binding.PageBlocks([binding.Pages(b[0], b[1]) for b in s["cache"]]) if own else None
        return s
    s["masks"] = torch.tensor([m for ps in parents for m in _bits(ps, case["words"])] + [[0] * case["words"]] * case["pad"], dtype=torch.int64, device="cuda")
    heads = case["heads"]
    s["q"] = _normal(gen, (cap, heads, dim), _DT[case["q"]])
    s["out"] = torch.zeros((cap, heads, dim), dtype=_DT[case["q"]], device="cuda")
    s["pages"] = binding.Pages(s["cache"][0, 0], s["cache"][0, 1]) if own else None
    s["workspace"] = binding.paged_attention_workspace(s["pages"], heads, _DT[case["q"]]) if own else None
    return s


def _prepare_verify(s, gen, flat, start):
    """Logits as language models give them: a few likely tokens over a wide floor, some tokens that are ruled out, and a draft that is near the target. The
    drafted tokens are drawn from the draft's probabilities at their parent, or are the draft's most likely ones there."""
    case, cap = s["case"], s["cap"]
    n, vocab, dtype = case["requests"], case["vocab"], _DT[case["dtype"]]
    stride = vocab + case["gap"]
    r = random.Random(case["seed0"] + 1)
    temperature = [0.0 if r.random() < case["greedy"] else r.uniform(0.5, 1.2) for _ in range(n)]
    s["temperature"] = torch.tensor(temperature, device="cuda")
    base = torch.randn((cap, stride), generator=gen, device="cuda") * 1.5
    few = min(16, vocab)
    likely = torch.randint(vocab, (cap, few), generator=gen, device="cuda")
    base.scatter_(1, likely, torch.randn((cap, few), generator=gen, device="cuda") * 2.5 + math.log(vocab))
    ruled_out = torch.randint(vocab, (max(1, vocab // 100),), generator=gen, device="cuda")
    keep = torch.randint(vocab, (1,), generator=gen, device="cuda")
    s["logits"] = base.to(dtype)
    s["logits"][:, ruled_out[ruled_out != keep]] = -math.inf
    s["logits"] = s["logits"][:, :vocab]
    draft = (base + torch.randn((cap, stride), generator=gen, device="cuda") * 0.7).to(dtype)[:, :vocab]
    del base
    above = [start[q] + p if p >= 0 else -1 for q in range(n) for p in flat[start[q]:start[q + 1]]]
    order, seen = [], {}
    for a in above:                                             # how many earlier siblings a row has
        order.append(seen.get(a, 0))
        seen[a] = order[-1] + 1
    parent = torch.tensor([max(a, 0) for a in above], device="cuda")
    tokens = torch.randint(vocab, (cap,), generator=gen, device="cuda")
    if case["drawn"]:
        t = torch.tensor([max(temperature[q], 1e-4) for q in range(n) for _ in range(start[q], start[q + 1])], device="cuda")
        for a in range(0, s["total"], 64):
            p = draft[parent[a:a + 64]].float() / t[a:a + 64, None]
            tokens[a:min(a + 64, s["total"])] = (p - torch.rand(p.shape, generator=gen, device="cuda").clamp(min=1e-30).log().neg().log()).argmax(-1)
        s["draft_logits"] = draft
    else:
        best = torch.topk(draft.float(), min(max(order) + 1, vocab), -1).indices
        tokens[:s["total"]] = best[parent, torch.tensor(order, device="cuda").clamp(max=best.shape[1] - 1)]
        s["draft_logits"] = None
    s["tokens"] = tokens.to(torch.int32)
    s["u_accept"], s["u_next"] = _uniform(gen, cap), _uniform(gen, n)
    s["path"] = torch.full((cap,), -1, dtype=torch.int32, device="cuda")
    s["n_path"], s["next_token"] = _int32([0] * n), _int32([0] * n)


# ---------------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _padded(s):
    """Row of the packed batch for each (request, row), and whether there is one."""
    start = s["row_start"].long()
    i = torch.arange(s["most_rows"], device=start.device)[None]
    return (start[:-1, None] + i).clamp(max=s["cap"] - 1), i < (start[1:] - start[:-1])[:, None]


def _packed(s, padded, into):
    """The packed batch back from (request, row); rows behind the last request stay as they were."""
    start = s["row_start"].long()
    t = torch.arange(s["cap"], device=start.device)
    request = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=start.numel() - 2)
    rows = padded[request, (t - start[request]).clamp(max=s["most_rows"] - 1)]
    live = (t < start[-1]).view(-1, *[1] * (rows.dim() - 1))
    into.copy_(torch.where(live, rows.to(into.dtype), into))
    return into


def _plan(s):
    row, live = _padded(s)
    n, m = row.shape
    words = s["case"]["words"]
    up = torch.where(live, s["parents"][row].long(), -1)
    seen = torch.eye(m, dtype=torch.bool, device=row.device).expand(n, m, m)
    depth = (up >= 0).long()
    for _ in range(max(1, (m - 1).bit_length())):               # ancestors of ancestors, twice as far each time
        at = up.clamp(min=0)
        there = up >= 0
        seen = seen | (seen.gather(1, at[:, :, None].expand(n, m, m)) & there[:, :, None])
        depth = depth + torch.where(there, depth.gather(1, at), 0)
        up = torch.where(there, up.gather(1, at), -1)
    cached = s["kv_len"] - (s["row_start"][1:] - s["row_start"][:-1])
    wide = torch.zeros((n, m, words * 64), dtype=torch.int64, device=row.device)
    wide[:, :, :m] = seen
    masks = (wide.view(n, m, words, 64) << torch.arange(64, device=row.device)).sum(-1)
    return dict(positions=_packed(s, cached[:, None] + depth, s["positions"]), masks=_packed(s, masks, s["masks"]))


def _tree(s):
    c = s["case"]
    heads, kv_heads, dim, page = c["heads"], c["kv_heads"], c["dim"], c["page"]
    groups = heads // kv_heads
    row, live = _padded(s)
    n, m = row.shape
    used = -(-s["longest"] // page)
    table = s["block_table"][:, :used].clamp(min=0).long()
    k, v = (s["cache"][0, i][table].float().permute(0, 2, 1, 3, 4).reshape(n, kv_heads, used * page, dim) for i in range(2))
    length = used * page
    cached = (s["kv_len"] - (s["row_start"][1:] - s["row_start"][:-1])).long()
    bits = (s["masks"][row][..., None] >> torch.arange(64, device=row.device)) & 1
    bits = bits.view(n, m, -1).bool()                           # [request][row][new row]
    at = torch.arange(length, device=row.device)[None] - cached[:, None]
    new = at.clamp(0, bits.shape[2] - 1)[:, None].expand(n, m, length)
    sees = (at[:, None] < 0) | ((at[:, None] <= torch.arange(m, device=row.device)[None, :, None]) & bits.gather(2, new))
    q = s["q"].float()[row].view(n, m, kv_heads, groups, dim).permute(0, 2, 1, 3, 4).reshape(n, kv_heads, m * groups, dim) * dim ** -0.5
    score = (q @ k.transpose(-1, -2).contiguous()).view(n, kv_heads, m, groups, length)
    score = score.masked_fill_(~sees[:, None, :, None], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    p = score.div_(score.sum(-1, keepdim=True)).view(n, kv_heads, m * groups, length)
    out = (p @ v).view(n, kv_heads, m, groups, dim).permute(0, 2, 1, 3, 4).reshape(n, m, heads, dim)
    return _packed(s, out, s["out"])


def _probabilities(logits, temperature):
    """Rows of probabilities in 64 bits; of a temperature of 0: all on the first of the largest."""
    x = logits.double()
    top, first = x.max(-1, keepdim=True)[0], x.argmax(-1, keepdim=True)
    e = ((x - top) / temperature.double()[:, None].clamp(min=1e-300)).exp()
    one = torch.zeros_like(x).scatter_(1, first, 1.0)
    return torch.where(temperature[:, None] == 0, one, e / e.sum(-1, keepdim=True))


def _verify(s):
    """All requests side by side, row after row: a row whose parent is the node reached so far is tried."""
    row, live = _padded(s)
    n, m = row.shape
    temperature = s["temperature"]
    parents, tokens, u = s["parents"][row], s["tokens"][row].long(), s["u_accept"].double()[row]
    here = torch.arange(n, device=row.device)
    node = torch.zeros(n, dtype=torch.long, device=row.device)
    drawn = s["draft_logits"] is not None
    p = _probabilities(s["logits"][row[:, 0]], temperature)
    q = _probabilities(s["draft_logits"][row[:, 0]], temperature) if drawn else torch.zeros_like(p)
    taken, left = torch.zeros(n, dtype=torch.float64, device=row.device), torch.ones(n, dtype=torch.float64, device=row.device)
    count = live[:, 0].long()
    path = torch.full((n, m + 1), -1, dtype=torch.long, device=row.device)
    path[:, 0] = torch.where(live[:, 0], 0, -1)
    for j in range(1, m):
        tried = live[:, j] & (parents[:, j] == node)
        px, qx = p[here, tokens[:, j]], q[here, tokens[:, j]]
        good = tried & (px > ((taken + u[:, j] * left) * qx if drawn else u[:, j] * left))
        bad = tried & ~good & (qx > 0 if drawn else True)       # (a token that the draft cannot have drawn says nothing about its distribution)
        if drawn:
            taken = torch.where(bad, taken + left, taken)
            left = torch.where(bad, (p - taken[:, None] * q).clamp(min=0).sum(-1), left)
            q = torch.where(good[:, None], _probabilities(s["draft_logits"][row[:, j]], temperature), q)
        else:
            left = torch.where(bad, left - px, left)
            p[here, tokens[:, j]] = torch.where(bad, 0.0, px)
        p = torch.where(good[:, None], _probabilities(s["logits"][row[:, j]], temperature), p)
        taken, left = torch.where(good, 0.0, taken), torch.where(good, 1.0, left)
        node = torch.where(good, j, node)
        path[here, torch.where(good, count, m)] = torch.where(good, j, -1)
        count = count + good
    w = (p - taken[:, None] * q).clamp(min=0) if drawn else p
    upto = torch.cumsum(w, -1)
    past = upto > s["u_next"].double()[:, None] * upto[:, -1:]
    s["next_token"].copy_(torch.where(live[:, 0], past.int().argmax(-1), -1))
    s["n_path"].copy_(count)
    return dict(path=_packed(s, path[:, :m], s["path"]), n_path=s["n_path"], next_token=s["next_token"])


def _keep(s):
    page, table, cache = s["case"]["page"], s["block_table"].long(), s["cache"]
    row, live = _padded(s)
    n, m = row.shape
    cached = (s["kv_len"] - (s["row_start"][1:] - s["row_start"][:-1])).long()
    j = torch.arange(m, device=row.device)[None].expand(n, m)
    kept = live & (j < s["n_path"][:, None])
    to = cached[:, None] + torch.where(kept, j, 0)              # what is not kept repeats the root's move, from its place to its place
    come = cached[:, None] + torch.where(kept, s["path"][row].long(), 0)
    to, come = to.reshape(-1), come.reshape(-1)
    request = torch.arange(n, device=row.device)[:, None].expand(n, m).reshape(-1)
    values = cache[:, :, table[request, come // page], :, come % page]
    cache[:, :, table[request, to // page], :, to % page] = values
    s["cached"].copy_(cached + s["n_path"])
    return dict(cache=cache, cached=s["cached"])


# ---------------------------------------------------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------------------------------------------------
def _own(s, kind):
    from paper_2505_16162_amd import binding
    if kind == "plan":
        binding.knnssd_tree_plan(s["parents"], s["row_start"], s["kv_len"], s["positions"], s["masks"])
        return dict(positions=s["positions"], masks=s["masks"])
    if kind == "tree":
        return binding.knnssd_tree_attention(s["pages"], s["block_table"], s["row_start"], s["kv_len"], s["masks"], s["q"], s["workspace"], out=s["out"],
                                             most_rows=s["most_rows"])
    if kind == "verify":
        path, n_path, next_token = binding.knnssd_tree_verify(
            s["logits"], s["tokens"], s["parents"], s["row_start"], s["temperature"], s["u_accept"], s["u_next"], s["workspace"], draft_logits=s["draft_logits"],
            path=s["path"], n_path=s["n_path"], next_token=s["next_token"], most_children=s["most_children"])
        return dict(path=path, n_path=n_path, next_token=next_token)
    binding.knnssd_tree_keep(s["blocks"], s["block_table"], s["row_start"], s["kv_len"], s["path"], s["n_path"], s["cached"])
    return dict(cache=s["cache"], cached=s["cached"])


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _own(s, kind)
    return {"plan": _plan, "tree": _tree, "verify": _verify, "keep": _keep}[kind](s)


def work(case):
    parents, cached, paths = _structure(case)
    rows = [len(p) for p in parents]
    total = sum(rows)
    if case["kind"] == "plan":
        return dict(bytes=total * (4 + 4 + 8 * case["words"]) + 8 * len(rows), flops=0)
    if case["kind"] == "verify":
        inner = sum(len(set(p) - {-1}) for p in parents) if case["drawn"] else 0
        values = (total + inner) * case["vocab"]
        return dict(bytes=values * (4 if case["dtype"] == "fp32" else 2) + 16 * total, flops=3 * values)
    kvb = 4 if case["kv"] == "fp32" else 2
    if case["kind"] == "keep":
        moved = sum(1 for p in paths for j, i in enumerate(p) if i != j)
        return dict(bytes=moved * case["blocks"] * 2 * case["kv_heads"] * case["dim"] * kvb * 2 + 16 * len(rows), flops=0)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    qb = 4 if case["q"] == "fp32" else 2
    seen = sum(len(p) * b + sum(bin(m).count("1") for m in _masks(p)) for p, b in zip(parents, cached))      # (row, position) pairs
    lens = sum(a + b for a, b in zip(rows, cached) if a)
    return dict(bytes=2 * total * heads * dim * qb + 2 * lens * kv_heads * dim * kvb + 8 * case["words"] * total, flops=4 * seen * heads * dim)


def _masks(parents):
    got = []
    for i, p in enumerate(parents):
        got.append((got[p] if p >= 0 else 0) | 1 << i)
    return got


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_tree(s):
    c = s["case"]
    heads, dim, page = c["heads"], c["dim"], c["page"]
    groups = heads // c["kv_heads"]
    out = s["out"].double()
    start, parents = s["row_start"].tolist(), s["parents"].tolist()
    for r, (a, b) in enumerate(zip(start, start[1:])):
        if a == b:
            continue
        length = s["kv_len"][r].item()
        cached = length - (b - a)
        sees = torch.zeros((b - a, length), dtype=torch.bool)
        sees[:, :cached] = True
        for i in range(b - a):
            j = i
            while j >= 0:                                       # up to the root
                sees[i, cached + j] = True
                j = parents[a + j]
        sees = sees.cuda()
        at = torch.arange(length, device="cuda")
        pages = s["block_table"][r, at // page].long()
        k, v = s["cache"][0, 0][pages, :, at % page], s["cache"][0, 1][pages, :, at % page]
        for h in range(heads):
            score = s["q"][a:b, h].double() @ k[:, h // groups].double().t().contiguous() / math.sqrt(dim)
            out[a:b, h] = torch.softmax(score.masked_fill(~sees, -math.inf), -1) @ v[:, h // groups].double()
    return out


def _softmax64(x, t):
    x = x.double()
    if t == 0:
        return torch.zeros_like(x).index_fill_(0, x.argmax(), 1.0)
    return torch.softmax(x / t, 0)


def _exact_verify(s):
    """Request by request, the target's distribution made anew after each rejection."""
    start, parents, tokens = s["row_start"].tolist(), s["parents"].tolist(), s["tokens"].tolist()
    u, u_next, temperature = s["u_accept"].double().tolist(), s["u_next"].double().tolist(), s["temperature"].double().tolist()
    path, counts, nexts = [-1] * s["cap"], [], []
    for r, (a, b) in enumerate(zip(start, start[1:])):
        if a == b:
            counts.append(0)
            nexts.append(-1)
            continue
        kept, node = [0], 0
        while True:
            p = _softmax64(s["logits"][a + node], temperature[r])
            children = [i for i in range(node + 1, b - a) if parents[a + i] == node]
            q = _softmax64(s["draft_logits"][a + node], temperature[r]) if s["draft_logits"] is not None and children else None
            went = None
            for i in children:
                x = tokens[a + i]
                drawn_from = q if q is not None else torch.zeros_like(p).index_fill_(0, torch.tensor(x, device="cuda"), 1.0)
                if u[a + i] * drawn_from[x] < p[x]:
                    went = i
                    break
                if drawn_from[x] == 0:                          # the draft cannot have drawn it
                    continue
                rest = (p - drawn_from).clamp(min=0) if q is not None else torch.where(drawn_from > 0, 0.0, p)
                p = rest / rest.sum()
            if went is None:
                break
            node = went
            kept.append(node)
        upto = torch.cumsum(p, 0)
        nexts.append(int((upto > u_next[r] * upto[-1]).int().argmax()))
        path[a:a + len(kept)] = kept
        counts.append(len(kept))
    return dict(path=_int32(path), n_path=_int32(counts), next_token=_int32(nexts))


def exact(case, seed):
    s = prepare(case, seed)
    start = s["row_start"].tolist()
    if case["kind"] == "tree":
        return _exact_tree(s)
    if case["kind"] == "verify":
        return _exact_verify(s)
    parents = s["parents"].tolist()
    if case["kind"] == "plan":
        positions, masks, lens = s["positions"].tolist(), s["masks"].tolist(), s["kv_len"].tolist()
        for r, (a, b) in enumerate(zip(start, start[1:])):
            depth = []
            for i in range(b - a):
                p = parents[a + i]
                depth.append(depth[p] + 1 if p >= 0 else 0)
                positions[a + i] = lens[r] - (b - a) + depth[i]
            masks[a:b] = _bits(parents[a:b], case["words"])
        return dict(positions=_int32(positions), masks=torch.tensor(masks, dtype=torch.int64, device="cuda"))
    page, table, path, lens, counts = case["page"], s["block_table"].tolist(), s["path"].tolist(), s["kv_len"].tolist(), s["n_path"].tolist()
    cache = s["cache"].clone()
    cached = []
    for r, (a, b) in enumerate(zip(start, start[1:])):
        base = lens[r] - (b - a)
        for j in range(counts[r]):
            to, come = base + j, base + path[a + j]
            cache[:, :, table[r][to // page], :, to % page] = s["cache"][:, :, table[r][come // page], :, come % page]
        cached.append(base + counts[r])
    return dict(cache=cache, cached=_int32(cached))
