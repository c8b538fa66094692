"""knnssd_tree_keep against lists."""
import random

import pytest
import torch

from paper_2505_16162_amd import binding

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32


class KeepCase:
    def __init__(self, rows, cached, paths, kv_heads, dim, page, dtype, n_blocks, order="head", seed=0, pad=2):
        g = torch.Generator().manual_seed(seed)
        n = len(rows)
        lens = [a + b for a, b in zip(rows, cached)]
        need = [-(-v // page) for v in lens]
        self.page, self.n_blocks = page, n_blocks
        n_pages, width = sum(need) + 2, max(need) + 1
        ids = torch.randperm(n_pages, generator=g).tolist()
        self.table = [[ids.pop() if j < need[r] else 2 ** 30 for j in range(width)] for r in range(n)]
        shape = (n_blocks, 2, n_pages, kv_heads, page, dim) if order == "head" else (n_blocks, 2, n_pages, page, kv_heads, dim)
        values = torch.randn(shape, generator=g).to(dtype)
        self.cache = values.cuda() if order == "head" else values.cuda().permute(0, 1, 2, 4, 3, 5)
        self.before = self.cache.cpu()
        self.rows, self.cached, self.paths, self.lens = rows, cached, paths, lens
        start = [0]
        for a in rows:
            start.append(start[-1] + a)
        flat = [v for p, a in zip(paths, rows) for v in (p + [-1] * a)[:a]] + [0] * pad
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.blocks = binding.PageBlocks([binding.Pages(b[0], b[1]) for b in self.cache])
        self.args = [ints(self.table), ints(start), ints(lens), ints(flat), ints([len(p) for p in paths])]
        self.out = ints([-9] * n)

    def want(self):
        cache, cached = self.before.clone(), []
        for r, path in enumerate(self.paths):
            base, kept, last = self.lens[r] - self.rows[r], 0, -1
            for j, i in enumerate(path[:self.rows[r]]):
                if i <= last or i >= self.rows[r]:
                    break
                to, come = base + j, base + i
                cache[:, :, self.table[r][to // self.page], :, to % self.page] = self.before[:, :, self.table[r][come // self.page], :, come % self.page]
                kept, last = j + 1, i
            cached.append(base + kept)
        return cache, cached

    def check(self):
        binding.knnssd_tree_keep(self.blocks, *self.args, self.out)
        cache, cached = self.want()
        assert self.out.tolist() == cached
        got = self.cache.cpu()
        assert torch.equal(got.view(torch.int16), cache.view(torch.int16))


def some_path(rng, n):
    return [] if n == 0 else [0] + sorted(rng.sample(range(1, n), rng.randint(0, n - 1)))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("kv_heads,dim,page,order,n_blocks", [(1, 64, 8, "head", 1), (8, 128, 16, "head", 3), (3, 64, 16, "position", 2), (40, 128, 64, "position", 2), (5, 128, 32, "head", 1),
                                                              (2, 64, 8, "head", 70)])
def test_paths(dtype, kv_heads, dim, page, order, n_blocks):
    rng = random.Random(kv_heads)
    rows = [1, 26, 0, 64, 5, 9]
    KeepCase(rows, [3, 100, 7, 0, 31, page], [some_path(rng, n) for n in rows], kv_heads, dim, page, dtype, n_blocks, order).check()


@pytest.mark.parametrize("path", [[0], [], [0, 1, 2, 3, 4, 5], [0, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11], [0, 1, 3, 5, 7, 9, 11], [5], [1, 2, 3], [11], list(range(1, 12))])
def test_entries_that_go_where_others_come_from(path):
    KeepCase([12], [13], [path], 2, 64, 8, BF16, 2).check()


def test_a_long_path():
    KeepCase([1024], [100], [list(range(0, 1024, 2))], 1, 64, 16, FP32, 1).check()
    KeepCase([1024], [0], [[0] + list(range(2, 1024))], 1, 64, 1024, BF16, 1).check()


@pytest.mark.parametrize("path", [[0, 3, 3, 5], [0, 5, 4], [-1, 2], [0, 12], [0, 2 ** 31 - 1], [0, 4, -2 ** 31, 7], [0, 0], [3, 1]])
def test_a_path_ends_before_an_entry_that_is_none(path):
    KeepCase([12], [13], [path], 2, 64, 8, BF16, 1).check()


def test_counts_that_are_none():
    for count, want in ((-5, 13), (2 ** 31 - 1, 25)):
        c = KeepCase([12], [13], [list(range(12))], 2, 64, 8, BF16, 1)
        c.args[4].fill_(count)
        binding.knnssd_tree_keep(c.blocks, *c.args, c.out)
        assert c.out.tolist() == [want] and torch.equal(c.cache.cpu(), c.before)


def test_tables_and_lengths_that_are_wrong():
    """Nothing that is no page is read or written; entries beyond the table end the path."""
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    c = KeepCase([12, 5], [13, 4], [[0, 2, 5], [0, 3]], 2, 64, 8, BF16, 1)
    table, start, lens, path, count = c.args
    binding.knnssd_tree_keep(c.blocks, torch.full_like(table, -1), start, lens, path, count, c.out)
    assert torch.equal(c.cache.cpu(), c.before) and c.out.tolist() == [16, 6]
    for wrong, want in (([2 ** 31 - 1, -7], [2 ** 31 - 13, 0]), ([11, 4], [0, 0])):
        binding.knnssd_tree_keep(c.blocks, table, start, ints(wrong), path, count, c.out)
        assert torch.equal(c.cache.cpu(), c.before) and c.out.tolist() == want
    for wrong in ([-2 ** 31, 2 ** 31 - 1, 3], [100, 200, 300], [12, 5, 5]):
        binding.knnssd_tree_keep(c.blocks, table * 0, ints(wrong), lens, path, count, c.out)
        torch.cuda.synchronize()


def test_refusals():
    c = KeepCase([12], [13], [[0, 2]], 2, 64, 8, BF16, 2)
    for out in (c.args[2], c.args[4]):
        with pytest.raises(binding.KnnSsdError) as e:
            binding.knnssd_tree_keep(c.blocks, *c.args, out)
        assert e.value.code == -1
    other = KeepCase([12], [13], [[0, 2]], 2, 64, 16, BF16, 1)
    with pytest.raises(binding.KnnSsdError) as e:
        binding.knnssd_tree_keep(binding.PageBlocks(c.blocks.blocks + other.blocks.blocks), *c.args, c.out)
    assert e.value.code == -2
    with pytest.raises(ValueError):
        binding.knnssd_tree_keep(c.blocks, *c.args, c.out.long())
