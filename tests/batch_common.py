"""Plain forms of the batch calls in 64 bits, their inputs, and the errors that their types allow."""
import math

import torch

EPS32 = 2.0 ** -24                      # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Stack:
    """Pages of a batch as lists: what knnssd_page_plan does, request by request."""

    def __init__(self, n_requests, width, n_pages, page):
        self.table = [[-1] * width for _ in range(n_requests)]
        self.held = [0] * n_requests
        self.free = list(range(n_pages - 1, -1, -1))
        self.n_pages, self.page, self.width = n_pages, page, width

    def plan(self, cached, added, max_rows):
        lens = [c + a for c, a in zip(cached, added)]
        need = [-(-v // self.page) for v in lens]
        back = sum(max(0, h - n) for h, n in zip(self.held, need))
        take = sum(max(0, n - h) for h, n in zip(self.held, need))
        n = len(lens)
        wrong = 0
        if any(c < 0 or a < 0 for c, a in zip(cached, added)):
            wrong = 1
        elif sum(added) > max_rows:
            wrong = 2
        elif any(v > self.width for v in need):
            wrong = 3
        elif take > len(self.free) + back:
            wrong = 4
        if wrong:
            return dict(row_start=[0] * (n + 1), kv_len=[0] * n, slots=[-1] * max_rows, positions=[-1] * max_rows, result=[0, 0, wrong, 0])
        before = len(self.free)
        for r in reversed(range(n)):
            while self.held[r] > need[r]:
                self.held[r] -= 1
                self.free.append(self.table[r][self.held[r]])
                self.table[r][self.held[r]] = -1
        for r in range(n):
            while self.held[r] < need[r]:
                self.table[r][self.held[r]] = self.free.pop()
                self.held[r] += 1
        start, slots, positions = [0], [], []
        for r in range(n):
            start.append(start[-1] + added[r])
            positions += range(cached[r], lens[r])
            slots += [self.table[r][p // self.page] * self.page + p % self.page for p in range(cached[r], lens[r])]
        pad = [-1] * (max_rows - len(slots))
        return dict(row_start=start, kv_len=lens, slots=slots + pad, positions=positions + pad, result=[start[-1], before - len(self.free), 0, max(lens)])


def attend64(q, k, v, scale, weights_dtype=None):
    """q [n][H][d], k and v [L][Hkv][d] (row i at position L - n + i): outputs in 64 bits, and per output the error that fp32 scores and sums, and
    weights rounded to weights_dtype, may make. With e = the largest error of a scaled score (d products and sums of half a step each,
    two more products), a weight is off by 2e relative to the row's sum at most, its exponential by four half steps more, and the sums of L
    weights and products by L half steps; all of it relative to sum(p |v|). A rounding of the weights adds its half step."""
    n, heads, d = q.shape
    length, group = k.shape[0], heads // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out = torch.zeros_like(q)
    err = torch.zeros_like(q)
    for i in range(n):
        seen = length - n + i + 1
        if seen <= 0:
            continue
        for h in range(heads):
            kk, vv = k[:seen, h // group], v[:seen, h // group]
            s = (kk @ q[i, h]) * scale
            p = torch.softmax(s, 0)
            out[i, h] = p @ vv
            e = ((kk.abs() @ q[i, h].abs()).max() * abs(scale)) * (d + 4) * EPS32
            err[i, h] = (p @ vv.abs()) * (2 * e + (2 * seen + 8) * EPS32 + (half_step(weights_dtype) if weights_dtype else 0.0))
    return out, err


class PagedCase:
    """Pages, tables and queries of a batch. Whatever no row sees holds NaN: page tails, pages of nobody, table entries beyond a request's."""

    def __init__(self, rows, lens, heads, kv_heads, dim, page, q_dtype, kv_dtype, order="head", pad=3, seed=0, device="cuda", gap=0):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.lens, self.heads, self.kv_heads, self.dim = rows, lens, heads, kv_heads, dim
        n, total = len(rows), sum(rows)
        need = [-(-v // page) for v in lens]
        width = max(1, max(need)) + 2
        n_pages = sum(need) + 3
        ids = torch.randperm(n_pages, generator=g).tolist()
        self.table = torch.full((n, width), -7, dtype=torch.int32)
        self.table[:, -1] = 2 ** 30
        k = torch.full((n_pages, kv_heads, page, dim), math.nan)
        v = torch.full((n_pages, kv_heads, page, dim), math.nan)
        self.k, self.v = [], []
        for r in range(n):
            kr = torch.randn(lens[r], kv_heads, dim, generator=g).to(kv_dtype)
            vr = torch.randn(lens[r], kv_heads, dim, generator=g).to(kv_dtype)
            self.k.append(kr)
            self.v.append(vr)
            for j in range(need[r]):
                at = ids.pop()
                self.table[r, j] = at
                m = min(page, lens[r] - j * page)
                k[at, :, :m] = kr[j * page:j * page + m].permute(1, 0, 2).float()
                v[at, :, :m] = vr[j * page:j * page + m].permute(1, 0, 2).float()
        k, v = k.to(device, kv_dtype), v.to(device, kv_dtype)
        if order == "position":
            k, v = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (k, v))
        self.k_pages, self.v_pages = k, v
        start = [0]
        for a in rows:
            start.append(start[-1] + a)
        self.start = start
        self.row_start = torch.tensor(start, dtype=torch.int32, device=device)
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device=device)
        self.block_table = self.table.to(device)
        cap = total + pad
        whole = torch.randn(cap, heads + gap, dim, generator=g).to(q_dtype).to(device)
        self.q = whole[:, :heads]
        self.out = torch.full((cap, heads + gap, dim), 5.0, dtype=q_dtype, device=device)[:, :heads]

    def want(self, scale, weights_dtype):
        q = self.q.cpu()
        outs, errs = [], []
        for r, (a, b) in enumerate(zip(self.start, self.start[1:])):
            o, e = attend64(q[a:b], self.k[r], self.v[r], scale, weights_dtype)
            outs.append(o)
            errs.append(e)
        return torch.cat(outs), torch.cat(errs)


def check_rows(got, want, err, dtype, pad_value=5.0):
    """Every value within err and the rounding of dtype; rows behind the last request's as they were."""
    got = got.cpu().double()
    n = want.shape[0]
    assert torch.isfinite(got).all()
    off = (got[:n] - want).abs() - (err + half_step(dtype) * (want.abs() + err))
    worst = off.max().item() if off.numel() else 0.0
    assert worst <= 0, (worst, (off > 0).nonzero()[:4].tolist())
    assert (got[n:] == pad_value).all()
