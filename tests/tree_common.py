"""Plain forms of the calls for trees of drafted tokens, in 64 bits on the CPU, and their inputs."""
import math
import random

import torch

import batch_common as B


def make_parents(rng, n, shape="tree"):
    """Parents of n rows: a chain, a star, a tree, or several trees side by side."""
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "star":
        return [-1] + [0] * (n - 1)
    return [-1] * min(n, 1) + [-1 if shape == "forest" and rng.random() < 0.2 else rng.randrange(max(0, i // 2 - 2), i) for i in range(1, n)]


def plan(parents, words):
    """(depths, masks as sets) of one request; parents that are no earlier row are none."""
    depth, seen = [], []
    for i, p in enumerate(parents):
        p = p if 0 <= p < i else -1
        depth.append(depth[p] + 1 if p >= 0 else 0)
        seen.append((seen[p] if p >= 0 else set()) | {i})
    return depth, seen


def bits(sets, words):
    """Masks as rows of signed 64-bit words."""
    out = torch.zeros(len(sets), words, dtype=torch.int64)
    for i, s in enumerate(sets):
        for w in range(words):
            v = sum(1 << (j - 64 * w) for j in s if w * 64 <= j < w * 64 + 64)
            out[i, w] = v - (1 << 64) if v >= 1 << 63 else v
    return out


def attend64(q, k, v, scale, sees, weights_dtype=None):
    """batch_common.attend64 for rows that see the positions `sees` [rows][positions] says: (result, the error that a calculation in fp32 with weights rounded to
    weights_dtype may make), by the same arithmetic."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, err = torch.zeros_like(q), torch.zeros_like(q)
    for h in range(heads):
        kk, vv = k[:, h // group], v[:, h // group]
        score = (q[:, h] @ kk.t()) * scale
        p = torch.softmax(score.masked_fill(~sees, -math.inf), -1)
        p = torch.where(sees.any(-1, keepdim=True), p, 0.0)
        out[:, h] = p @ vv
        e = ((q[:, h].abs() @ kk.abs().t()) * sees).amax(-1, keepdim=True) * abs(scale) * (d + 4) * B.EPS32
        err[:, h] = (p @ vv.abs()) * (2 * e + (2 * sees.sum(-1, keepdim=True) + 8) * B.EPS32 + (B.half_step(weights_dtype) if weights_dtype else 0.0))
    return out, err


def weights64(x, temperature):
    """softmax's numerators: at even logits whole numbers, so that a border at a round number stays one."""
    x = x.double()
    if temperature == 0:
        return torch.zeros_like(x).index_fill_(0, (x == x.max()).nonzero()[0], 1.0)
    return torch.exp((x - x.max()) / temperature)


def softmax64(x, temperature):
    w = weights64(x, temperature)
    return w / w.sum()


def bad(x):
    return bool(torch.isnan(x).any() or (x == math.inf).any() or (x == -math.inf).all())


def verify(logits, draft, tokens, parents, temperature, u, u_next):
    """(path, next token) of one request. Its rows' logits [rows][vocab]; what is left of p is made anew, as probabilities, after each rejection."""
    n = len(tokens)
    if n == 0 or not 0 <= temperature < math.inf:
        return [], -1
    path, node, vocab = [0], 0, logits.shape[1]
    while True:
        children = [i for i in range(node + 1, n) if parents[i] == node and 0 <= tokens[i] < vocab]
        if bad(logits[node]) or (draft is not None and children and bad(draft[node])):
            return path, -1
        p, rest = softmax64(logits[node], temperature), weights64(logits[node], temperature)
        q = softmax64(draft[node], temperature) if draft is not None and children else None
        went = None
        for i in children:
            x = tokens[i]
            of = q if q is not None else torch.zeros_like(p).index_fill_(0, torch.tensor([x]), 1.0)
            if p[x] > u[i] * of[x]:
                went = i
                break
            if of[x] == 0:
                continue
            p = (p - of).clamp(min=0) if q is not None else torch.where(of > 0, 0.0, p)
            rest = p if q is not None else torch.where(of > 0, 0.0, rest)
            if p.sum() == 0:
                break
            p = p / p.sum()
        if went is None:
            break
        node = went
        path.append(node)
    upto = torch.cumsum(rest, 0)
    if not upto[-1] > 0:
        return path, -1
    past = ((upto > u_next * upto[-1]) & (rest > 0)).nonzero()
    return path, int(past[0] if len(past) else (rest > 0).nonzero()[-1])


class VerifyCase:
    """Logits, drafted tokens and numbers of a batch, on the CPU. Behind a row's vocabulary, in rows behind the last request's and in the draft's rows that nobody draws from: NaN."""

    def __init__(self, rows, vocab, dtype, drawn, shape="tree", temperatures=(0.7,), pad=2, gap=0, seed=0, likely=6):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.rows, self.vocab, self.drawn, self.dtype = rows, vocab, drawn, dtype
        total = sum(rows)
        self.total, self.cap = total, total + pad
        self.start = [0]
        for a in rows:
            self.start.append(self.start[-1] + a)
        self.temperature = torch.tensor([temperatures[r % len(temperatures)] for r in range(len(rows))]).double().tolist()      # (the call gets fp32)
        base = torch.randn(total, vocab, generator=g)
        few = torch.randint(vocab, (total, min(likely, vocab)), generator=g)
        base.scatter_(1, few, torch.randn(few.shape, generator=g) * 2 + math.log(vocab))
        self.wide = torch.full((self.cap, vocab + gap), math.nan, dtype=dtype)
        self.wide[:total, :vocab] = base.to(dtype)
        self.logits = self.wide[:, :vocab]
        self.wide_draft = torch.full((self.cap, vocab + gap), math.nan, dtype=dtype)
        self.parents = [p for a in rows for p in make_parents(rng, a, shape)]
        draft = (base + 0.7 * torch.randn(total, vocab, generator=g)).to(dtype)
        self.tokens = []
        taken = {}
        for r, a in enumerate(rows):
            for i in range(a):
                p = self.parents[self.start[r] + i]
                row = self.start[r] + max(p, 0)
                if drawn:
                    self.wide_draft[row, :vocab] = draft[row]
                    pr = softmax64(draft[row], self.temperature[r])
                    self.tokens.append(int(torch.multinomial(pr, 1, generator=g)))
                else:
                    best = draft[row].float().argsort(descending=True)
                    k = taken.get(row, 0) if i else 0
                    taken[row] = k + (1 if i else 0)
                    self.tokens.append(int(best[min(k, vocab - 1)]))
        self.draft = self.wide_draft[:, :vocab] if drawn else None
        self.u = torch.rand(self.cap, generator=g)
        self.u_next = torch.rand(len(rows), generator=g)

    def want(self):
        path, counts, nexts = [], [], []
        for r, (a, b) in enumerate(zip(self.start, self.start[1:])):
            p, t = verify(self.logits[a:b], None if self.draft is None else self.draft[a:b], self.tokens[a:b], self.parents[a:b], self.temperature[r],
                          self.u[a:b].double().tolist(), float(self.u_next[r].double()))
            path += p + [-1] * (b - a - len(p))
            counts.append(len(p))
            nexts.append(t)
        return path, counts, nexts

    def on_gpu(self):
        """Arguments of binding.knnssd_tree_verify, but for the workspace."""
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        pad = [0] * (self.cap - self.total)
        wide, wide_draft = self.wide.cuda(), self.wide_draft.cuda()
        return dict(logits=wide[:, :self.vocab], tokens=ints(self.tokens + pad), parents=ints(self.parents + pad), row_start=ints(self.start),
                    temperature=torch.tensor(self.temperature, device="cuda"), u_accept=self.u.cuda(), u_next=self.u_next.cuda(),
                    draft_logits=wide_draft[:, :self.vocab] if self.drawn else None)
