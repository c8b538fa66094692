"""The batch calls together, as a program that serves several requests uses them: a decoder whose products are plain torch, its prompts through
knnssd_prompt_attention, its rounds of drafts verified over pages, against the library's own single-request decoding; and a context's cache read as pages."""
import pytest
import torch

import batch_common as B
from paper_2505_16162_amd import binding, synth

pytestmark = pytest.mark.gpu


class BatchDecoder:
    """The full model for a batch of requests. Only what depends on which row is whose goes through the library."""

    def __init__(self, shape, weights, n_requests, max_rows, page_size, stream=None):
        dev = "cuda"
        move = lambda t: t.to(dev).float()  # noqa: E731
        self.s = shape
        self.embed, self.head, self.final = move(weights["embed"]), move(weights["lm_head"]), move(weights["final_norm"])
        self.blocks = [dict(qkv=torch.cat([move(b["wq"]), move(b["wk"]), move(b["wv"])]), o=move(b["wo"]), g=move(b["wg"]), u=move(b["wu"]), d=move(b["wd"]),
                            an=move(b["attn_norm"]), mn=move(b["mlp_norm"])) for b in weights["blocks"]]
        n_pages = n_requests * -(-shape.max_seq // page_size)
        kv = torch.float32 if shape.kv_dtype == "fp32" else torch.bfloat16
        self.pages = [binding.Pages.empty(n_pages, page_size, shape.n_kv_heads, shape.head_dim, kv) for _ in self.blocks]
        self.tables = binding.PageTables.fresh(n_requests, shape.max_seq, n_pages, page_size)
        self.rows = binding.BatchRows(n_requests, max_rows)
        self.ws = binding.paged_attention_workspace(self.pages[0], shape.n_heads, torch.float32)
        self.max_rows = max_rows

    def norm(self, x, g):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.s.rms_eps) * g

    def forward(self, tokens, cached, added, prompts=False):
        """Arg-max tokens of the rows of all requests (tokens: one list, request behind request)."""
        s, ints = self.s, lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        binding.knnssd_page_plan(self.tables, self.rows, ints(cached), ints(added))
        ids = torch.zeros(self.max_rows, dtype=torch.long, device="cuda")
        ids[:len(tokens)] = torch.tensor(tokens, device="cuda")
        x = self.embed[ids]
        q_out = torch.zeros(self.max_rows, s.n_heads, s.head_dim, device="cuda")
        k_out = torch.zeros(self.max_rows, s.n_kv_heads, s.head_dim, device="cuda")
        for b, pages in zip(self.blocks, self.pages):
            qkv = self.norm(x, b["an"]) @ b["qkv"].t()
            binding.knnssd_paged_store(pages, qkv, self.rows.slots, self.rows.positions, s.rope_base, q_out, k_out if prompts else None)
            if prompts:
                v = qkv.view(self.max_rows, -1, s.head_dim)[:, -s.n_kv_heads:]
                att = binding.knnssd_prompt_attention(q_out, k_out, v, self.rows.row_start, out=torch.zeros_like(q_out))
            else:
                att = binding.knnssd_paged_attention(pages, self.tables.block_table, self.rows.row_start, self.rows.kv_len, q_out, self.ws,
                                                     out=torch.zeros_like(q_out), most_rows=max(added))
            x = x + att.reshape(self.max_rows, -1) @ b["o"].t()
            h = self.norm(x, b["mn"])
            x = x + (torch.nn.functional.silu(h @ b["g"].t()) * (h @ b["u"].t())) @ b["d"].t()
        assert self.rows.result[2].item() == 0
        return (self.norm(x, self.final) @ self.head.t()).argmax(-1)[:len(tokens)].tolist()


@pytest.mark.parametrize("kv_heads", [4, 2])
def test_rounds_of_drafts_for_several_requests(kv_heads):
    """Three requests of different lengths at once; drafts of different counts, some wrong, so that requests accept different numbers and give pages back.
    Every request's tokens are those that the library decodes for it alone (an fp32 model: the two differ by fp32 rounding)."""
    shape = synth.small_shape("batch", n_kv_heads=kv_heads, max_seq=128, weight_dtype="fp32", kv_dtype="fp32")
    weights = synth.make_weights(shape, seed=5, gains="random", std=0.05)
    prompts = [synth.make_prompt(shape.vocab, n, seed=n).tolist() for n in (7, 33, 20)]
    new = 24
    gpu = binding.KnnSsd(shape, weights)
    want = [gpu.knnssd_generate(p, new, 0)[0] for p in prompts]
    gpu.close()
    dec = BatchDecoder(shape, weights, 3, 70, 8)
    lens = [len(p) for p in prompts]
    first = dec.forward(sum(prompts, []), [0, 0, 0], lens, prompts=True)
    out = [[first[sum(lens[:r + 1]) - 1]] for r in range(3)]
    cached = list(lens)
    rounds = 0
    while any(len(o) < new for o in out):
        drafts = []
        for r in range(3):
            k = 0 if len(out[r]) >= new else min((rounds + 2 * r) % 5, new - 1 - len(out[r]))
            d = want[r][len(out[r]):len(out[r]) + k]
            if (rounds + r) % 3 == 0 and len(d) > 1:
                d[1] = (d[1] + 1) % shape.vocab               # a wrong draft
            drafts.append(d)
        live = [len(out[r]) < new for r in range(3)]
        added = [1 + len(d) if a else 0 for d, a in zip(drafts, live)]
        got = dec.forward(sum(([out[r][-1]] + drafts[r] for r in range(3) if live[r]), []), cached, added)
        at = 0
        for r in range(3):
            if not live[r]:
                continue
            mine, at = got[at:at + added[r]], at + added[r]
            j = 0
            while j < len(drafts[r]) and drafts[r][j] == mine[j]:
                j += 1
            out[r] += mine[:j + 1]
            cached[r] += j + 1
        rounds += 1
        assert rounds < 60
    assert [o[:new] for o in out] == want
    binding.knnssd_page_plan(dec.tables, dec.rows, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert dec.tables.n_free.item() == dec.tables.free_pages.numel() and sorted(dec.tables.free_pages.tolist()) == list(range(dec.tables.free_pages.numel()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("generic", [False, True])
def test_a_contexts_cache_as_pages(dtype, generic):
    """Several continuations of one prompt at once over the cache that knnssd_prefill wrote: each reads the same pages."""
    shape = synth.small_shape("pages_" + dtype, n_kv_heads=2, d_ffn=704, max_seq=96, weight_dtype=dtype, kv_dtype=dtype)
    gpu = binding.KnnSsd(shape, synth.make_weights(shape, seed=3, gains="random", std=0.05), generic_kernels=generic)
    prompt = synth.make_prompt(shape.vocab, 53, seed=8).tolist()
    gpu.knnssd_prefill(prompt)
    torch.cuda.synchronize()
    t = torch.float32 if dtype == "fp32" else torch.bfloat16
    for block in range(shape.n_blocks):
        pages = gpu.knnssd_context_pages(block, 32)
        assert pages.k.shape == (3, 2, 32, 64) and pages.k.dtype == t
        kv = [gpu.knnssd_read_kv(block, p) for p in range(53)]
        k, v = (torch.stack([x[i] for x in kv]).view(53, 2, 64) for i in range(2))
        q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(block)).to(t)
        table = torch.tensor([[0, 1]] * 3, dtype=torch.int32, device="cuda")
        start = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
        lens = torch.tensor([53, 40, 1], dtype=torch.int32, device="cuda")
        out = binding.knnssd_paged_attention(pages, table, start, lens, q.cuda(), binding.paged_attention_workspace(pages, 4, t))
        both = [B.attend64(q[i:i + 1], k[:n], v[:n], 0.125, torch.bfloat16 if dtype == "bf16" else None) for i, n in enumerate((53, 40, 1))]
        B.check_rows(out, torch.cat([o for o, _ in both]), torch.cat([e for _, e in both]), t)
    for block, page, code in ((-1, 32, -3), (shape.n_blocks, 32, -3), (0, 64, -2), (0, 24, -2), (0, 4, -2)):
        with pytest.raises(binding.KnnSsdError) as e:
            gpu.knnssd_context_pages(block, page)
        assert e.value.code == code
    gpu.close()
