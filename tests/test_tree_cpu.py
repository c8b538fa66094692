"""Trees of drafted tokens without a GPU: refusals, which come in front of the first launch, and what the plain form that the GPU is held to says about distributions."""
import ctypes
import itertools
import random

import pytest
import torch

import tree_common as T
from paper_2505_16162_amd import binding
from test_batch_cpu import BAD_PAGES, pages

OK, EINVAL, ESHAPE, ERANGE = 0, -1, -2, -3
A = 0x100000            # an address that nothing dereferences


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def call(fn, base, kw):
    assert set(kw) <= set(base)
    return fn(*[v for v in {**base, **kw}.values()])


PLAN = dict(parents=A, row_start=A, kv_len=A, n=2, rows=5, positions=2 * A, masks=3 * A, words=1, stream=None)
ATTENTION = dict(pages=None, table=A, width=4, row_start=A, kv_len=A, n=2, masks=A, words=1, q=A, qs=4 * 128, out=2 * A, os=4 * 128, dtype=1, rows=5, heads=4, scale=0.1,
                 most=0, ws=A, wsb=1 << 40, stream=None)
VERIFY = dict(logits=A, ls=1000, draft=A, ds=1000, dtype=1, vocab=1000, tokens=A, parents=A, row_start=A, n=2, rows=5, temperature=A, u=A, u_next=A, path=2 * A, n_path=3 * A,
              next_token=4 * A, most=0, ws=A, wsb=1 << 40, stream=None)
KEEP = dict(blocks=None, n_blocks=2, table=A, width=4, row_start=A, kv_len=A, n=2, rows=5, path=A, n_path=2 * A, cached=3 * A, stream=None)


@pytest.mark.parametrize("kw,code", [(dict(parents=None), EINVAL), (dict(row_start=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(positions=None), EINVAL),
                                     (dict(masks=None), EINVAL), (dict(masks=A + 4), EINVAL), (dict(words=0), ERANGE), (dict(words=17), ERANGE), (dict(words=-1), ERANGE),
                                     (dict(n=0), ERANGE), (dict(n=4097), ERANGE), (dict(rows=0), ERANGE), (dict(rows=2 ** 23 + 1), ERANGE),
                                     (dict(positions=A), EINVAL), (dict(positions=A - 16), EINVAL), (dict(masks=A + 8), EINVAL), (dict(kv_len=2 * A - 4), EINVAL),
                                     (dict(positions=3 * A + 36), EINVAL), (dict(row_start=3 * A + 32), EINVAL)])
def test_plan(lib, kw, code):
    assert call(lib.knnssd_tree_plan, PLAN, kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(masks=None), EINVAL), (dict(masks=A + 4), EINVAL), (dict(words=0), ERANGE), (dict(words=17), ERANGE), (dict(table=None), EINVAL), (dict(kv_len=None), EINVAL),
    (dict(row_start=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(ws=None), EINVAL), (dict(ws=A + 16), EINVAL), (dict(wsb=0), EINVAL), (dict(q=A + 8), EINVAL),
    (dict(qs=4 * 128 - 8), EINVAL), (dict(dtype=3), EINVAL), (dict(n=0), ERANGE), (dict(rows=0), ERANGE), (dict(width=0), ERANGE), (dict(most=-1), ERANGE),
    (dict(scale=float("nan")), ERANGE), (dict(heads=3), ESHAPE), (dict(rows=2 ** 23 + 1), ERANGE)])
def test_attention(lib, kw, code):
    p = pages()
    assert call(lib.knnssd_tree_attention, dict(ATTENTION, pages=ctypes.byref(p)), kw) == code


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_pages_of_attention_and_keep(lib, kw, code):
    p = pages(**kw)
    assert call(lib.knnssd_tree_attention, ATTENTION, dict(pages=ctypes.byref(p))) == code
    assert call(lib.knnssd_tree_keep, KEEP, dict(blocks=(binding.PagesStruct * 2)(p, p))) == code


@pytest.mark.parametrize("kw,code", [(dict([(k, None)]), EINVAL) for k in ("logits", "tokens", "parents", "row_start", "temperature", "u", "u_next", "path", "n_path", "next_token", "ws")] + [
    (dict(dtype=2), EINVAL), (dict(vocab=0), ESHAPE), (dict(vocab=-5), ESHAPE), (dict(vocab=2 ** 19 + 1, ls=2 ** 20, ds=2 ** 20), ESHAPE), (dict(ls=999), EINVAL), (dict(ds=999), EINVAL),
    (dict(ls=-1000), EINVAL), (dict(logits=A + 1), EINVAL), (dict(draft=A + 1), EINVAL), (dict(dtype=0, logits=A + 2), EINVAL), (dict(dtype=0, draft=A + 2), EINVAL), (dict(n=0), ERANGE),
    (dict(n=4097), ERANGE), (dict(rows=0), ERANGE), (dict(rows=2 ** 23 + 1), ERANGE), (dict(rows=2 ** 20, vocab=152064, ls=152064, ds=152064), ERANGE), (dict(most=-1), ERANGE),
    (dict(ws=A + 128), EINVAL), (dict(wsb=255), EINVAL), (dict(path=A), EINVAL), (dict(path=A - 16), EINVAL), (dict(n_path=A + 16), EINVAL), (dict(next_token=A + 4), EINVAL),
    (dict(tokens=4 * A - 16), EINVAL), (dict(u_next=3 * A + 4), EINVAL), (dict(n_path=2 * A + 16), EINVAL), (dict(next_token=3 * A - 4), EINVAL)])
def test_verify(lib, kw, code):
    assert call(lib.knnssd_tree_verify, VERIFY, kw) == code


def test_workspace_of_the_verification(lib):
    f = lib.knnssd_tree_verify_bytes
    assert f(5, 2, 1000, 0) > 0 and f(5, 2, 1000, 1) > f(5, 2, 1000, 0)
    assert f(50, 2, 2049, 0) > f(50, 2, 2048, 0)
    for bad in ((0, 2, 1000, 1), (5, 0, 1000, 1), (5, 4097, 1000, 1), (5, 2, 0, 1), (5, 2, 2 ** 19 + 1, 1), (2 ** 23, 2, 152064, 1)):
        assert f(*bad) == 0
    # a workspace for drafts that were not drawn is too small for drawn ones
    assert call(lib.knnssd_tree_verify, VERIFY, dict(wsb=f(5, 2, 1000, 0))) == EINVAL
    with pytest.raises(binding.KnnSsdError):
        binding.tree_verify_workspace(5, 2, 2 ** 20, True, "cpu")


@pytest.mark.parametrize("kw,code", [(dict(table=None), EINVAL), (dict(row_start=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(path=None), EINVAL), (dict(n_path=None), EINVAL),
                                     (dict(cached=None), EINVAL), (dict(n_blocks=0), ERANGE), (dict(n_blocks=1025), ERANGE), (dict(width=0), ERANGE), (dict(n=0), ERANGE),
                                     (dict(n=4097), ERANGE), (dict(rows=0), ERANGE), (dict(cached=A), EINVAL), (dict(cached=A + 4), EINVAL), (dict(cached=2 * A - 4), EINVAL),
                                     (dict(cached=5 * A, path=5 * A - 16), EINVAL), (dict(cached=5 * A, row_start=5 * A - 8), EINVAL),
                                     (dict(cached=5 * A, table=5 * A - 28), EINVAL)])
def test_keep(lib, kw, code):
    blocks = (binding.PagesStruct * 2)(pages(), pages(k_dev=3 * A, v_dev=4 * A))
    assert call(lib.knnssd_tree_keep, dict(KEEP, blocks=blocks), kw) == code


@pytest.mark.parametrize("kw", [dict(), dict(k_dev=3 * A), dict(v_dev=3 * A), dict(k_dev=2 * A, v_dev=3 * A), dict(k_dev=3 * A, v_dev=3 * A)])
def test_keep_refuses_a_cache_that_is_given_twice(lib, kw):
    """It would be moved twice: blocks that share their caches are given once, keys and values are two."""
    assert call(lib.knnssd_tree_keep, dict(KEEP, blocks=(binding.PagesStruct * 2)(pages(), pages(**kw))), {}) == EINVAL


def test_keep_wants_blocks_alike(lib):
    assert call(lib.knnssd_tree_keep, KEEP, {}) == EINVAL
    for kw in (dict(n_pages=11), dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=64), dict(pos_stride=256), dict(head_stride=32 * 128), dict(page_stride=8 * 16 * 128)):
        both = (binding.PagesStruct * 2)(pages(), pages(**kw))
        assert call(lib.knnssd_tree_keep, KEEP, dict(blocks=both)) == ESHAPE, kw


def test_the_binding_refuses_tensors_of_other_places():
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(ValueError, match="on a GPU"):
        binding.knnssd_tree_plan(i, i, i, i, torch.zeros(4, 1, dtype=torch.int64))
    with pytest.raises(ValueError, match="on a GPU"):
        binding.knnssd_tree_verify(torch.zeros(4, 9), i, i, i, f, f, f, f)
    with pytest.raises(ValueError, match="one GPU"):
        binding.PageBlocks([])


def outcome(p_logits, q_logits, tokens, parents, temperature):
    """Distribution of the token behind the root that comes out of a tree of depth one, over all numbers: each child's probability of being taken, which
    the plain form's walk has to have on its two sides."""
    vocab = p_logits.shape[1]
    p = T.softmax64(p_logits[0], temperature)
    got = torch.zeros(vocab, dtype=torch.float64)
    left, weight = p, 1.0
    q = None if q_logits is None else T.softmax64(q_logits[0], temperature)
    for i in range(1, len(tokens)):
        x = tokens[i]
        of = q if q is not None else torch.zeros_like(p).index_fill_(0, torch.tensor([x]), 1.0)
        pass_ = float((left[x] / of[x]).clamp(max=1.0))
        # the plain form's walk goes on to this child for numbers below that probability, and for no others
        for u, taken in ((pass_ * (1 - 1e-9), True), (pass_ * (1 + 1e-9) + 1e-15, False)):
            if u > 0 and u < 0.99999:
                path, _ = T.verify(p_logits, q_logits, tokens[:i + 1], parents[:i + 1], temperature, [0.999999999] * i + [u], 0.5)
                assert path == ([0, i] if taken else [0])
        got[x] += weight * pass_
        weight *= 1 - pass_
        if weight < 1e-12:
            return got
        rest = (left - of).clamp(min=0) if q is not None else torch.where(of > 0, 0.0, left)
        left = rest / rest.sum()
    return got + weight * left


@pytest.mark.parametrize("temperature", [1.0, 0.6])
@pytest.mark.parametrize("children", [1, 2, 3])
def test_what_comes_out_has_the_models_distribution(temperature, children):
    """All draws of up to three children from q, each with its probability: the first token is distributed as p."""
    g = torch.Generator().manual_seed(children)
    vocab = 4
    p_logits, q_logits = torch.randn(children + 1, vocab, generator=g), torch.randn(children + 1, vocab, generator=g)
    p, q = T.softmax64(p_logits[0], temperature), T.softmax64(q_logits[0], temperature)
    got = torch.zeros(vocab, dtype=torch.float64)
    for xs in itertools.product(range(vocab), repeat=children):
        chance = float(torch.stack([q[x] for x in xs]).prod())
        got += chance * outcome(p_logits, q_logits, [0, *xs], [-1] + [0] * children, temperature)
    assert (got - p).abs().max() < 1e-6
    # drafts that were not drawn: for any choice of them
    for xs in itertools.permutations(range(vocab), children):
        assert (outcome(p_logits, None, [0, *xs], [-1] + [0] * children, temperature) - p).abs().max() < 1e-6


def test_the_closed_form_of_what_is_left():
    """p after j rejections is max(p - c q, 0) / S with c += S, S = sum max(p - c q, 0): against one step after the other."""
    g = torch.Generator().manual_seed(1)
    p, q = torch.softmax(2 * torch.randn(50, generator=g).double(), 0), torch.softmax(2 * torch.randn(50, generator=g).double(), 0)
    left, c, s = p, 0.0, 1.0
    for _ in range(5):
        left = (left - q).clamp(min=0)
        left = left / left.sum()
        c += s
        s = float((p - c * q).clamp(min=0).sum())
        assert (left - (p - c * q).clamp(min=0) / s).abs().max() < 1e-12


def test_masks_of_the_plain_form():
    parents = T.make_parents(random.Random(3), 70)
    depth, seen = T.plan(parents, 2)
    assert depth[0] == 0 and all(depth[i] == len(seen[i]) - 1 for i in range(70))
    m = T.bits(seen, 2)
    assert all(bool(int(m[i, j // 64]) >> (j % 64) & 1) == (j in seen[i]) for i in range(70) for j in range(70))
