"""knnssd_tree_verify where numbers are 0 and probabilities next to nothing: against the plain form, on the CPU in 64 bits. Whole numbers: all have to be equal."""
import math

import pytest
import torch

import tree_common as T
from test_gpu_tree_verify import call

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


def counted(logits, temperature):
    """Logits of the tokens that count: those of 2^-500 of the row's largest weight and less are ruled out."""
    x = logits.double()
    return torch.where((x - x.max(-1, keepdim=True).values) / temperature > -500 * math.log(2), x, -math.inf)


def outcome(logits, tokens, parents, u, temperature, u_next, draft=None, rows=0):
    """One request on the GPU, in arrays of `rows` rows at least, which has to be the plain form's outcome for the tokens that count."""
    n = len(tokens)
    cap = max(n, rows)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    rowed = lambda x: torch.cat([x, x[:1].expand(cap - n, -1)]).cuda()  # noqa: E731
    args = dict(logits=rowed(logits), tokens=ints(list(tokens) + [0] * (cap - n)), parents=ints(list(parents) + [-1] * (cap - n)), row_start=ints([0, n]),
                temperature=torch.tensor([temperature], device="cuda"), u_accept=torch.tensor(list(u) + [0.0] * (cap - n), device="cuda"),
                u_next=torch.tensor([u_next], device="cuda"), draft_logits=None if draft is None else rowed(draft))
    path, n_path, next_token = call(args, cap, 1, logits.shape[1])
    t, u64 = torch.tensor(temperature).double().item(), [torch.tensor(x).double().item() for x in u]
    want = T.verify(counted(logits, t), None if draft is None else counted(draft, t), list(tokens), list(parents), t, u64, torch.tensor(u_next).double().item())
    assert (path.tolist()[:n_path.item()], next_token.item()) == want
    return want


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("temperature,gap", [(0.05, 16.0), (0.05, 18.0), (0.05, 25.0), (0.05, 36.0), (0.05, 40.0), (0.02, 6.5), (0.02, 10.0), (0.02, 14.0)])
@pytest.mark.parametrize("rows", [0, 2800])
def test_a_number_of_0_where_the_first_tokens_are_next_to_impossible(dtype, temperature, gap, rows):
    """The likely tokens are all in the vocabulary's second chunk of 2048; the others are `gap` below, 460 to 1150 powers of two. (2800 rows in bf16: the rows' sums by the table of powers.)"""
    g = torch.Generator().manual_seed(1)
    low = 8.0 - gap
    x = torch.full((3, 5000), low)
    x[:, 2060:4000:7] = 8.0 + (torch.randn(3, 278, generator=g).clamp(-3, 3) * 0.05)
    x = x.to(dtype)
    q = x.roll(7, 1)
    first = 0 if gap * math.log2(math.e) / temperature < 500 else 2060
    assert outcome(x, [0], [-1], [0.0], temperature, 0.0, rows=rows) == ([0], first)
    # behind a token that is given and rejected, behind one that is drawn and rejected, and behind a drawn one that is taken
    top = int(x[0].float().argmax())
    few = int(x[0].float().argsort(descending=True)[5])
    outcome(x, [0, few], [-1, 0], [0.0, 0.9999], temperature, 0.0, rows=rows)
    assert outcome(x, [0, 2060], [-1, 0], [0.0, 0.9999], temperature, 0.0, rows=rows) == ([0], 2067 if first else 0)
    outcome(x, [0, few], [-1, 0], [0.0, 0.9999], temperature, 0.0, q, rows=rows)
    assert outcome(x, [0, top], [-1, 0], [0.0, 0.0], temperature, 0.0, q, rows=rows) == ([0, 1], first)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("again", [2, 63, 64, 70, 200])
def test_a_token_of_next_to_no_probability_again_with_a_number_of_0(dtype, again):
    """A given draft of 10^-26 is tried once and rejected; what is left of p has nothing on its token, so no number takes it, not even 0, though the rest still sums up to 1 in 64 bits."""
    n = again + 2
    x = torch.tensor([[0.0, 60.0, 59.0, -math.inf]] * n).to(dtype)
    tokens, parents, u = [3] * n, [0] * n, [0.5] * n
    parents[0] = -1
    tokens[1] = tokens[again] = 0
    u[again] = 0.0
    tokens[again + 1] = 1
    assert outcome(x, tokens, parents, u, 1.0, 0.5) == ([0, again + 1], 1)
    assert outcome(x, tokens[:-1], parents[:-1], u[:-1], 1.0, 0.0) == ([0], 1)
