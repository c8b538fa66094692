"""knnssd_tree_verify against the plain form, which makes the distributions anew after each rejection, on the CPU in 64 bits. Whole numbers: all have to be equal."""
import math

import pytest
import torch

import tree_common as T
from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def call(args, n_rows, n_requests, vocab, fill=255, **kw):
    ws = binding.tree_verify_workspace(n_rows, n_requests, vocab, args["draft_logits"] is not None)
    ws.fill_(fill)
    return binding.knnssd_tree_verify(workspace=ws, **args, **kw)


def check(c, **kw):
    path, n_path, next_token = call(c.on_gpu(), c.cap, len(c.rows), c.vocab, path=torch.full((c.cap,), -9, dtype=torch.int32, device="cuda"), **kw)
    want = c.want()
    assert n_path.tolist() == want[1]
    assert path.tolist() == want[0] + [-9] * (c.cap - c.total)
    assert next_token.tolist() == want[2]
    return want


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("vocab,gap", [(1, 0), (2, 1), (7, 0), (255, 3), (1024, 0), (2048, 8), (2049, 0), (5001, 1), (32000, 0), (70001, 5)])
def test_sizes(dtype, drawn, vocab, gap):
    check(T.VerifyCase([1, 9, 0, 14, 5], vocab, dtype, drawn, temperatures=(0.8, 0.0, 1.3), gap=gap, seed=vocab))
    check(T.VerifyCase([6, 2], vocab, dtype, drawn, shape="chain", temperatures=(0.5, 1.0), gap=gap, seed=vocab + 1), most_children=1)


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("shape", ["chain", "star", "tree", "forest"])
@pytest.mark.parametrize("temperature", [0.0, 0.3, 1.0, 5.0])
def test_shapes_and_temperatures(drawn, shape, temperature):
    taken = 0
    for seed in range(6):
        c = T.VerifyCase([12, 3, 30], 600, FP32 if seed % 2 else BF16, drawn, shape, (temperature,), seed=seed, likely=3)
        for most in (0, 1, 3):                                # (a hint, right or wrong: the same result)
            want = check(c, most_children=most)
        taken += sum(want[1]) - 3
    assert taken > 0


@pytest.mark.parametrize("drawn", [False, True])
def test_many_rows(drawn):
    check(T.VerifyCase([1024, 300, 65], 120, BF16, drawn, "tree", seed=1))
    check(T.VerifyCase([1024], 40, FP32, drawn, "star", seed=2, likely=30, temperatures=(4.0,)))
    c = T.VerifyCase([200], 50, FP32, drawn, "chain", seed=3, likely=1, temperatures=(0.2,))
    c.u[:] = 0.0
    check(c)


@pytest.mark.parametrize("drawn", [False, True])
def test_many_requests(drawn):
    rows = [(i * 7) % 5 for i in range(700)]
    check(T.VerifyCase(rows, 90, BF16, drawn, "tree", (0.9, 0.0, 2.0), seed=4))


def test_rows_beyond_a_tree():
    """1100 rows: those from 1024 on are none of the tree."""
    c = T.VerifyCase([1100], 30, FP32, False, "star", seed=1, likely=25, temperatures=(3.0,))
    c.u[:1024] = 1.0 - 2.0 ** -24
    c.tokens[1:1024] = [c.tokens[1]] * 1023
    path, n_path, next_token = call(c.on_gpu(), c.cap, 1, 30)
    want, token = T.verify(c.logits[:1024], None, c.tokens[:1024], c.parents[:1024], 3.0, c.u[:1024].double().tolist(), float(c.u_next[0]))
    assert want == [0] and n_path.tolist() == [1] and path.tolist()[:1100] == [0] + [-1] * 1099 and next_token.tolist() == [token]


@pytest.mark.parametrize("drawn", [False, True])
@pytest.mark.parametrize("u,u_next", [(0.0, 0.0), (1.0 - 2.0 ** -24, 1.0 - 2.0 ** -24), (0.0, 1.0 - 2.0 ** -24), (1.0 - 2.0 ** -24, 0.0), (0.5, 0.5)])
def test_the_ends_of_the_numbers(drawn, u, u_next):
    for vocab in (40, 4500):
        c = T.VerifyCase([9, 1, 20], vocab, FP32, drawn, "tree", (0.7, 0.0), seed=3, likely=20)
        c.u[:], c.u_next[:] = u, u_next
        check(c)


def test_a_single_row_draws_a_token():
    """Every token has its share of the numbers: from the middle of each share that token comes, at both of its ends too (a step of fp32 inside)."""
    g = torch.Generator().manual_seed(2)
    for dtype, vocab in ((FP32, 33), (BF16, 300), (FP32, 2100)):
        row = (2 * torch.randn(vocab, generator=g)).to(dtype)
        row[::7] = -math.inf
        p = T.softmax64(row, 0.9)
        upto = torch.cumsum(p, 0)
        u, want = [], []
        for t in range(vocab):
            lo, hi = float(upto[t] - p[t]), float(upto[t])
            for x in (lo + (hi - lo) * f for f in (0.25, 0.5, 0.75)):
                x = torch.tensor(x, dtype=torch.float32).item()
                if lo + 1e-12 < x < hi - 1e-12:
                    u.append(x)
                    want.append(t)
        n = min(len(u), 4096)
        args = dict(logits=row.repeat(n, 1).cuda(), tokens=torch.zeros(n, dtype=torch.int32, device="cuda"), parents=torch.full((n,), -1, dtype=torch.int32, device="cuda"),
                    row_start=torch.arange(n + 1, dtype=torch.int32, device="cuda"), temperature=torch.full((n,), 0.9, device="cuda"), u_accept=torch.zeros(n, device="cuda"),
                    u_next=torch.tensor(u[:n], device="cuda"), draft_logits=None)
        # the temperature is the fp32 number that the call gets
        exact = T.softmax64(row, torch.tensor(0.9).double().item()).cumsum(0)
        keep = [i for i in range(n) if (exact - u[i]).abs().min() > 1e-12]
        path, n_path, next_token = call(args, n, n, vocab)
        got = next_token.tolist()
        assert [got[i] for i in keep] == [int((exact > u[i]).nonzero()[0]) for i in keep] and (n_path == 1).all() and (path == 0).all()


def one(logits, draft=None, tokens=(0,), parents=(-1,), temperature=1.0, u=None, u_next=0.5):
    """Outcome of one request on the GPU, which is the plain form's too."""
    n = len(tokens)
    u = [0.3] * n if u is None else u
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    args = dict(logits=logits.cuda(), tokens=ints(list(tokens)), parents=ints(list(parents)), row_start=ints([0, n]), temperature=torch.tensor([temperature], device="cuda"),
                u_accept=torch.tensor(u, device="cuda"), u_next=torch.tensor([u_next], device="cuda"), draft_logits=None if draft is None else draft.cuda())
    path, n_path, next_token = call(args, n, 1, logits.shape[1])
    got = path.tolist()[:n_path.item()], next_token.item()
    assert path.tolist()[n_path.item():] == [-1] * (n - n_path.item())
    t = torch.tensor(temperature).double().item()
    assert got == T.verify(logits, draft, list(tokens), list(parents), t, [torch.tensor(x).double().item() for x in u], torch.tensor(u_next).double().item())
    return got


@pytest.mark.parametrize("vocab", [5, 3000])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_values_that_are_no_numbers(vocab, dtype):
    g = torch.Generator().manual_seed(1)
    good = torch.randn(3, vocab, generator=g).to(dtype)
    for temperature in (1.0, 0.0):
        for value in (math.nan, math.inf):
            for at in (0, vocab - 1):
                x = good.clone()
                x[0, at] = value
                assert one(x, temperature=temperature) == ([0], -1)
                assert one(x, good, (0, 1), (-1, 0), temperature) == ([0], -1)
                assert one(good, x, (0, 1), (-1, 0), temperature) == ([0], -1)
                assert one(good, x, (0,), (-1,), temperature)[1] >= 0          # (nobody draws from it)
                # a row that is not reached, and one that is
                y = good.clone()
                y[1, at] = value
                top = int(good[0].float().argmax())
                low = int(good[0].float().argmin())
                assert one(y, None, (0, low), (-1, 0), temperature, u=[0.0, 0.9999])[1] >= 0
                assert one(y, None, (0, top), (-1, 0), temperature, u=[0.0, 0.0]) == ([0, 1], -1)
        x = good.clone()
        x[0] = -math.inf
        assert one(x, temperature=temperature) == ([0], -1)
        x[0, vocab - 1] = -3.0
        assert one(x, temperature=temperature) == ([0], vocab - 1)
    for temperature in (-1.0, math.nan, math.inf):
        assert one(good, temperature=temperature) == ([], -1)


def test_ruled_out_tokens():
    """-inf: never taken, never the next token, at any temperature."""
    x = torch.tensor([[-math.inf, 1.0, -math.inf, 0.5, -math.inf]] * 2)
    for temperature in (0.0, 1e-30, 1e-3, 1.0, 1e30):
        for u_next in (0.0, 0.4, 0.99999994):
            assert one(x, None, (0, 2), (-1, 0), temperature, u=[0.0, 0.0], u_next=u_next)[1] in (1, 3)
            assert one(x, x, (0, 2), (-1, 0), temperature, u=[0.0, 0.0], u_next=u_next)[1] in (1, 3)


def test_tokens_outside_the_vocabulary():
    x = torch.zeros(4, 6)
    for token in (-1, 6, 2 ** 31 - 1, -2 ** 31):
        assert one(x, None, (0, token, 3, token), (-1, 0, 0, 2), u=[0.0] * 4)[0] == [0, 2]
        assert one(x, x, (0, token, 3, token), (-1, 0, 0, 2), u=[0.0] * 4)[0] == [0, 2]
        assert one(x, None, (0, token), (-1, 0), u=[0.0] * 2)[0] == [0]


def test_the_same_token_again():
    x = torch.tensor([[2.0, 1.0, 0.0, -1.0]] * 5)
    # a draft that was not drawn is tried once: what is left of p has nothing on it
    assert one(x, None, (0, 0, 0, 0, 1), (-1, 0, 0, 0, 0), u=[0.0, 0.99, 0.0, 0.0, 0.0])[0] == [0, 4]
    assert one(x, None, (0, 0, 0, 0, 0), (-1, 0, 0, 0, 0), u=[0.0, 0.99, 0.0, 0.0, 0.0], u_next=0.0) == ([0], 1)
    q = torch.tensor([[0.0, 1.0, 2.0, 3.0]] * 5)
    for u in (0.01, 0.2, 0.9):
        one(x, q, (0, 3, 3, 3, 2), (-1, 0, 0, 0, 0), u=[0.0, u, u, u, u])


def test_a_distribution_with_nothing_left():
    """All tokens rejected one by one; p equal to q."""
    x = torch.tensor([[30.0, 0.0, -math.inf]] * 3)
    assert one(x, None, (0, 1, 0), (-1, 0, 0), u=[0.0, 0.9, 0.9]) == ([0, 2], 0)
    assert one(x, x, (0, 0), (-1, 0), u=[0.0, 0.99999994])[0] == [0, 1]
    assert one(x, x, (0, 2, 0), (-1, 0, 0), u=[0.0, 0.5, 0.99999994])[0] == [0, 2]      # (token 2 cannot have been drawn)


def test_greedy_ties_go_to_the_first():
    for vocab in (9, 6000):
        x = torch.zeros(2, vocab, dtype=BF16)
        x[0, 3::5] = 2.0
        assert one(x, None, (0, 3), (-1, 0), 0.0) == ([0, 1], 0)
        assert one(x, None, (0, 8), (-1, 0), 0.0) == ([0], 3)
        assert one(x, x, (0, 8), (-1, 0), 0.0) == ([0], 3)


def test_large_logits_and_steep_temperatures():
    g = torch.Generator().manual_seed(9)
    for size in (1e4, 1e30, 3e38):
        x = (torch.randn(3, 500, generator=g).clamp(-1, 1) * size).float()
        for temperature in (1e-3, 1.0, 1e10, 3e38):
            one(x, None, (0, 5, 7), (-1, 0, 1), temperature)
            one(x, x.flip(1).contiguous(), (0, 5, 7), (-1, 0, 1), temperature)


def test_the_same_call_gives_the_same_and_leaves_its_inputs():
    c = T.VerifyCase([30, 30, 9], 5000, FP32, True, "tree", seed=5)
    args = c.on_gpu()
    before = {k: v.clone() for k, v in args.items()}
    first = call(args, c.cap, 3, 5000)
    for fill in (0, 1, 127, 255):
        again = call(args, c.cap, 3, 5000, fill=fill)
        assert all(torch.equal(a[:c.total], b[:c.total]) for a, b in zip(first, again))
    for k, v in args.items():
        assert torch.equal(torch.nan_to_num(v.float(), nan=7.0), torch.nan_to_num(before[k].float(), nan=7.0))


def test_row_starts_that_are_wrong():
    """Bounded, not right: nothing outside the rows is written."""
    c = T.VerifyCase([9, 12], 300, FP32, True, "tree", seed=5, pad=0)
    args = c.on_gpu()
    whole = torch.full((60,), -9, dtype=torch.int32, device="cuda")
    for start in ([0, 2 ** 31 - 1, 5], [-2 ** 31, 9, 2 ** 31 - 1], [100, 200, 300], [9, 3, 21], [5, 5, 5]):
        args["row_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        call(args, 21, 2, 300, path=whole[20:41], n_path=whole[10:12], next_token=whole[50:52])
        torch.cuda.synchronize()
        assert all((whole[a:b] == -9).all() for a, b in ((0, 10), (12, 20), (41, 50), (52, 60)))


def test_refusals():
    c = T.VerifyCase([5], 300, FP32, True, pad=0)
    args = c.on_gpu()
    small = binding.tree_verify_workspace(5, 1, 300, False)
    with pytest.raises(binding.KnnSsdError):
        binding.knnssd_tree_verify(workspace=small[:-1], **args)
    for name, value in (("logits", args["logits"].t()), ("draft_logits", args["draft_logits"][:, :299]), ("draft_logits", args["draft_logits"].bfloat16()), ("logits", args["logits"][:4]),
                        ("logits", args["logits"].half()), ("tokens", args["tokens"].long()), ("parents", args["parents"][:4]), ("temperature", args["temperature"].double()),
                        ("u_accept", args["u_accept"][:4]), ("u_next", args["u_next"].cpu()), ("row_start", args["row_start"][:1])):
        with pytest.raises(ValueError):
            call({**args, name: value}, 5, 1, 300)
    with pytest.raises(ValueError):
        call(args, 5, 1, 300, path=args["tokens"][:4].clone())
