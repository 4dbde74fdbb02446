"""The operators as decoding uses them, step after step: pages for the last token and the drafts of each request, their keys and values into the pages, attention over the cache, verification, and the
rejected tokens taken off again.  The attention is held to chunk attention over the same tokens' keys and values laid out contiguously, tokens to the definition of the verification, pages to a stack.

Both attentions are within half a step of bf16 (2^-8 of the value) and some 2^-11 of the weighted sum of sizes of the same sums: chunk attention's weights go into products as one bf16 term (2^-8 of the
weighted sum of sizes at most), so they differ by less than 2^-7 |o| + 2^-7 sum(p |v|); values are below 5, so 2^-7 * 2 * 5 < 0.08 in any element, and in the 2-norm, where roundings
are independent, by 3 * 2^-8 < 1.2e-2 of the tensor."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc

pytestmark = pytest.mark.gpu
BF16, E4M3, I32, I64 = torch.bfloat16, torch.float8_e4m3fn, torch.int32, torch.int64


class Decoder:
    """n requests with a prompt each, a table of queries, keys and values in the place of a model's layers below, a matrix in the place of those above."""

    def __init__(self, n, drafts, page, kind, seed, heads=8, kv_heads=2, dim=64, vocab=61, width=40):
        from paper_2509_21275_amd import draft_verify as dv
        from paper_2509_21275_amd import paged_attn as pa
        from paper_2509_21275_amd import paged_cache as pc
        g = torch.Generator().manual_seed(seed)
        self.n, self.K, self.page, self.vocab, self.heads, self.kv_heads, self.dim, self.kind = n, drafts, page, vocab, heads, kv_heads, dim, kind
        self.scale = torch.full((kv_heads,), 2.0 ** -6, device="cuda") if kind == "e4m3" else None  # (a power of two: what 8 bits stand for is a bf16)

        def table(h):
            return torch.randn((vocab, h, dim), generator=g).to(BF16).cuda()

        self.q_of, self.k_of, self.v_of = table(heads), table(kv_heads), table(kv_heads)
        self.head = (0.3 * torch.randn((heads * dim, vocab), generator=g)).cuda()
        self.rng = torch.Generator().manual_seed(seed + 1)
        self.pages = n * width // 2
        self.cdesc = pc.make_desc(n, width, page, self.pages)
        rows = n * (1 + drafts)
        self.adesc = pa.make_desc(heads, kv_heads, dim, n, rows, page, self.pages, width, dim ** -0.5, kind)
        self.ws = pc.alloc_workspace(self.cdesc), pa.alloc_workspace(self.adesc), dv.alloc_workspace(n, drafts, vocab)
        z = lambda *s, dtype=I32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
        self.kv_len, self.held, self.table, self.num_free = z(n), z(n), z(n, width), torch.tensor([self.pages], dtype=I32, device="cuda")
        self.free = torch.randperm(self.pages, generator=g).to(I32).cuda()
        self.q_start, self.slots, self.granted = z(n + 1), z(rows, dtype=I64), z(n)
        self.caches = [torch.zeros((self.pages, kv_heads, page, dim), device="cuda").to(BF16 if kind == "bf16" else E4M3) for _ in range(2)]
        self.q, self.k, self.v, self.o = (torch.zeros((rows, h, dim), dtype=BF16, device="cuda") for h in (heads, kv_heads, kv_heads, heads))
        self.lse = torch.zeros((heads, rows), device="cuda")
        self.new = torch.full((n,), 1 + drafts, dtype=I32, device="cuda")
        self.target, self.draft = torch.zeros((n, drafts + 1, vocab), device="cuda"), torch.zeros((n, drafts, vocab), device="cuda")
        self.tokens, self.u, self.last_u = z(n, drafts), torch.zeros((n, drafts), device="cuda"), torch.zeros(n, device="cuda")
        self.accepted, self.rejected, self.out = z(n), z(n), z(n, drafts + 1)
        self.prompts = [torch.randint(0, vocab, (int(torch.randint(1, 60, (1,), generator=g)),), generator=g).tolist() for _ in range(n)]

    def prefill(self):
        """All prompts but their last tokens into the cache at once, as after a chunk's prefill."""
        from paper_2509_21275_amd import paged_cache as pc
        tokens = [t for p in self.prompts for t in p[:-1]]
        new = torch.tensor([len(p) - 1 for p in self.prompts], dtype=I32, device="cuda")
        slots, q_start = torch.zeros(max(1, len(tokens)), dtype=I64, device="cuda"), torch.zeros_like(self.q_start)
        pc.paged_cache_extend(self.cdesc, new, self.kv_len, self.held, self.table, self.free, self.num_free, self.kv_len, self.held, self.num_free, q_start, slots, None, self.ws[0])
        ids = torch.tensor(tokens, device="cuda", dtype=I64)
        pc.paged_cache_write(self.k_of[ids], self.v_of[ids], slots[:len(tokens)], *self.caches, self.scale, self.scale)

    def forward(self):
        """Pages, keys and values, attention."""
        from paper_2509_21275_amd import paged_attn as pa
        from paper_2509_21275_amd import paged_cache as pc
        pc.paged_cache_extend(self.cdesc, self.new, self.kv_len, self.held, self.table, self.free, self.num_free, self.kv_len, self.held, self.num_free, self.q_start, self.slots,
                              self.granted, self.ws[0])
        pc.paged_cache_write(self.k, self.v, self.slots, *self.caches, self.scale, self.scale)
        pa.paged_attn_fwd(self.adesc, self.q, *self.caches, self.table, self.kv_len, self.q_start, self.o, self.lse, self.ws[1], k_scale=self.scale, v_scale=self.scale)

    def choose(self):
        """Verification, and the rejected tokens off again."""
        from paper_2509_21275_amd import draft_verify as dv
        from paper_2509_21275_amd import paged_cache as pc
        dv.draft_verify(self.target, self.draft, self.tokens, None, self.u, self.last_u, self.accepted, self.rejected, self.out, self.ws[2])
        pc.paged_cache_truncate(self.cdesc, self.rejected, self.kv_len, self.held, self.table, self.free, self.num_free, self.kv_len, self.held, self.num_free, self.ws[0])

    def feed(self, last):
        """Drafts and random numbers of a step, queries, keys and values of [last token, drafts] of each request."""
        guess = torch.softmax(torch.randn((self.n, self.K, self.vocab), generator=self.rng), -1)
        self.tokens.copy_(torch.multinomial(guess.flatten(0, 1), 1, generator=self.rng).view(self.n, self.K).to(I32))
        self.draft.copy_(guess)
        self.u.copy_(torch.rand((self.n, self.K), generator=self.rng) * 0.5)
        self.last_u.copy_(torch.rand(self.n, generator=self.rng))
        ids = torch.cat((torch.tensor(last, dtype=I64)[:, None], self.tokens.cpu().long()), 1).flatten().cuda()
        for to, of in ((self.q, self.q_of), (self.k, self.k_of), (self.v, self.v_of)):
            to.copy_(of[ids])

    def logits(self):
        self.target.copy_(torch.softmax(self.o.float().flatten(1) @ self.head, -1).view(self.n, self.K + 1, self.vocab))

    def held_to_chunk_attention(self, texts):
        """o of the step against chunk attention over contiguous keys and values of texts + drafts."""
        import paper_2509_21275_amd as ca
        segs, ids, at, m = [], [], 0, 1 + self.K
        for i, t in enumerate(texts):
            whole = t + self.tokens[i].tolist()
            segs.append((i * m, m, at, len(whole)))
            ids += whole
            at += len(whole)
        ids = torch.tensor(ids, device="cuda")
        k, v = self.k_of[ids], self.v_of[ids]
        if self.kind == "e4m3":
            k, v = (((x.float() / self.scale[0]).clamp(-448, 448).to(E4M3).float() * self.scale[0]).to(BF16) for x in (k, v))
        desc = ca.make_desc(segs, self.heads, self.kv_heads, self.dim, self.n * m, at, self.dim ** -0.5)
        o, lse = torch.empty_like(self.q), torch.empty_like(self.lse)
        ca.chunk_attn_fwd(desc, self.q, k, v, o, lse, ca.alloc_workspace(desc))
        torch.cuda.synchronize()
        off = float((self.o.double() - o.double()).norm() / o.double().norm())
        assert off < 1.2e-2 and float((self.o.float() - o.float()).abs().max()) < 0.08, off
        # chunk attention of small chunks sums the weights as they are rounded to bf16, each by 2^-8 of itself at most, so that the logarithm of their sum is off by 2^-8 / (1 - 2^-8) < 4e-3;
        # the rest (scores of 64 products, below 40: 2^-24 * 72 * 40 on either side) is below 4e-4
        assert float((self.lse - lse).abs().max()) < 4.4e-3


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("n,drafts,page,kind", [(5, 3, 4, "bf16"), (7, 0, 16, "bf16"), (4, 5, 7, "e4m3"), (33, 2, 16, "e4m3")])
def test_decoding(n, drafts, page, kind, captured):
    d = Decoder(n, drafts, page, kind, seed=n)
    d.prefill()
    torch.cuda.synchronize()
    texts = [list(p) for p in d.prompts]
    assert d.kv_len.tolist() == [len(t) - 1 for t in texts]
    graphs = None
    if captured:
        d.feed([t[-1] for t in texts])
        state = [x.clone() for x in (d.kv_len, d.held, d.num_free, d.table, d.free)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs = []
        for f in (d.forward, d.choose):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                f()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(state, (d.kv_len, d.held, d.num_free, d.table, d.free)))
    for step in range(6):
        d.feed([t[-1] for t in texts])
        graphs[0].replay() if captured else d.forward()
        torch.cuda.synchronize()
        assert d.granted.all() and d.kv_len.tolist() == [len(t) + drafts for t in texts]
        d.held_to_chunk_attention(texts)
        d.logits()
        graphs[1].replay() if captured else d.choose()
        torch.cuda.synchronize()
        target, draft = d.target.double().cpu().numpy(), d.draft.double().cpu().numpy()
        for i, t in enumerate(texts):
            kept, out = orc.verify(target[i], draft[i], d.tokens[i].tolist(), drafts, d.u[i].tolist(), float(d.last_u[i]))
            assert d.accepted[i] == kept and d.out[i].tolist() == out, (step, i)
            t += out[:kept + 1]
        held = [-(-(len(t) - 1) // page) for t in texts]
        assert d.kv_len.tolist() == [len(t) - 1 for t in texts] and d.held.tolist() == held and int(d.num_free) == d.pages - sum(held)
        owned = [p for i in range(n) for p in d.table[i, :held[i]].tolist()] + d.free[:int(d.num_free)].tolist()
        assert sorted(owned) == list(range(d.pages))
    assert drafts == 0 or 0 < sum(len(t) - len(p) for t, p in zip(texts, d.prompts)) < 6 * n * (drafts + 1)
    # all requests end
    d.rejected.fill_(2**31 - 1)
    from paper_2509_21275_amd import paged_cache as pc
    pc.paged_cache_truncate(d.cdesc, d.rejected, d.kv_len, d.held, d.table, d.free, d.num_free, d.kv_len, d.held, d.num_free, d.ws[0])
    torch.cuda.synchronize()
    assert not d.kv_len.any() and not d.held.any() and sorted(d.free.tolist()) == list(range(d.pages))


def test_a_pool_that_runs_out():
    """Requests that find no pages are not served, and what they have stays right; when others end, they go on."""
    from paper_2509_21275_amd import paged_cache as pc
    n, page, width, pages = 6, 4, 8, 10
    desc = pc.make_desc(n, width, page, pages)
    z = lambda *s, dtype=I32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    kv_len, held, table, free, num_free = z(n), z(n), z(n, width), torch.arange(pages, dtype=I32, device="cuda"), torch.tensor([pages], dtype=I32, device="cuda")
    q_start, slots, granted, ws = z(n + 1), z(200, dtype=I64), z(n), pc.alloc_workspace(desc)
    rng, want = np.random.default_rng(0), (np.zeros(n, int), np.zeros(n, int), np.zeros((n, width), int), np.arange(pages), pages)
    refused = 0
    for step in range(40):
        new = rng.integers(0, 9, n)
        pc.paged_cache_extend(desc, torch.tensor(new, dtype=I32, device="cuda"), kv_len, held, table, free, num_free, kv_len, held, num_free, q_start, slots, granted, ws)
        a = orc.extend(page, pages, new, *want[:3], want[3], want[4], 200)
        refused += int((a[6] == 0).sum())
        drop = rng.integers(0, 12, n) * (rng.random(n) < 0.7)
        torch.cuda.synchronize()
        assert np.array_equal(slots.cpu().numpy(), a[5]) and np.array_equal(granted.cpu().numpy(), a[6])
        pc.paged_cache_truncate(desc, torch.tensor(drop, dtype=I32, device="cuda"), kv_len, held, table, free, num_free, kv_len, held, num_free, ws)
        b = orc.truncate(page, drop, a[0], a[1], a[2], want[3], a[3])
        want = (b[0], b[1], a[2], b[2], b[3])
        torch.cuda.synchronize()
        for x, y in zip((kv_len, held, table, num_free), (b[0], b[1], a[2], [b[3]])):
            assert np.array_equal(x.cpu().numpy(), y), step
        assert free[:b[3]].tolist() == b[2][:b[3]].tolist()
    assert refused > 10


class Refusing(Decoder):
    """The same where the pool may run out: a request that is not served, or has nothing new, has no drafts in the cache, and nothing is taken off it."""

    def __init__(self, *args, **kw):
        super().__init__(*args, **kw)
        self.count, self.idle = torch.zeros(self.n, dtype=I32, device="cuda"), set()

    def feed(self, last):
        """Rows of requests that have ended are not there: those of the others follow each other."""
        super().feed(last)
        at = [i * (1 + self.K) + j for i in range(self.n) if i not in self.idle for j in range(1 + self.K)]
        for x in (self.q, self.k, self.v):
            x[:len(at)] = x[at].clone()

    def choose(self):
        from paper_2509_21275_amd import draft_verify as dv
        from paper_2509_21275_amd import paged_cache as pc
        torch.mul(self.new - 1, self.granted, out=self.count)
        dv.draft_verify(self.target, self.draft, self.tokens, self.count, self.u, self.last_u, self.accepted, self.rejected, self.out, self.ws[2])
        pc.paged_cache_truncate(self.cdesc, self.rejected, self.kv_len, self.held, self.table, self.free, self.num_free, self.kv_len, self.held, self.num_free, self.ws[0])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_decoding_where_some_are_refused(kind):
    """What a refused request has in the cache stays, and it goes on from there when others have ended."""
    from paper_2509_21275_amd import paged_cache as pc
    n, drafts, page = 6, 3, 4
    d = Refusing(n, drafts, page, kind, seed=11, width=60)
    d.prefill()
    d.num_free.fill_(9)  # a step takes up to n of them
    torch.cuda.synchronize()
    texts, refused, again = [list(p) for p in d.prompts], set(), set()
    idle = d.idle
    for step in range(24):
        d.feed([t[-1] for t in texts])
        d.forward()
        torch.cuda.synchronize()
        granted = d.granted.tolist()
        served = [i for i in range(n) if granted[i] and i not in idle]
        waiting = [i for i in range(n) if not granted[i]]
        refused |= set(waiting)
        again |= refused & set(served)
        assert d.kv_len.tolist() == [0 if i in idle else len(t) + drafts if granted[i] else len(t) - 1 for i, t in enumerate(texts)]
        starts = d.q_start.tolist()
        for i in served:  # (in float64: a few rows)
            whole = torch.tensor(texts[i] + d.tokens[i].tolist(), device="cuda")
            k, v = d.k_of[whole].double(), d.v_of[whole].double()
            if kind == "e4m3":
                s = float(d.scale[0])
                k, v = ((x / s).float().clamp(-448, 448).to(E4M3).double() * s for x in (k, v))
            for j in range(1 + drafts):
                row, seen = starts[i] + j, len(texts[i]) + j
                x = torch.matmul(d.q[row].double().view(d.kv_heads, -1, d.dim), k[:seen].permute(1, 2, 0).contiguous()) * d.dim ** -0.5
                want = torch.matmul(torch.softmax(x, -1), v[:seen].transpose(0, 1).contiguous()).reshape(d.heads, d.dim)
                # half a step of bf16, and 2^-11 of values below 5
                assert float((d.o[row].double() - want).abs().max()) < 2.0 ** -8 * 5 + 2.0 ** -11 * 5, (step, i, j)
        d.target.copy_(torch.softmax(d.o.float().flatten(1) @ d.head, -1).view(n, drafts + 1, d.vocab))
        if idle:  # (their rows are not there, so that those of the others lie further ahead)
            at = torch.tensor([starts[i] for i in range(n)], device="cuda")
            rows = (at[:, None] + torch.arange(drafts + 1, device="cuda")).clamp(max=n * (drafts + 1) - 1)
            d.target.copy_(d.target.flatten(0, 1)[rows])
        before = [x.clone() for x in (d.kv_len, d.held, d.table)]
        d.choose()
        torch.cuda.synchronize()
        for i in waiting:
            assert d.rejected[i] == 0 and all(torch.equal(x[i], y[i]) for x, y in zip((d.kv_len, d.held, d.table), before)), (step, i)
        target, draft = d.target.double().cpu().numpy(), d.draft.double().cpu().numpy()
        for i in served:
            kept, out = orc.verify(target[i], draft[i], d.tokens[i].tolist(), drafts, d.u[i].tolist(), float(d.last_u[i]))
            assert d.accepted[i] == kept and d.out[i].tolist() == out, (step, i)
            texts[i] += out[:kept + 1]
        assert all(d.kv_len[i] == len(texts[i]) - 1 for i in range(n) if i not in idle)
        if len(waiting) > 1 and len(idle) < 3:  # one of those that were served ends
            i = served[0]
            idle.add(i)
            drop = torch.zeros_like(d.rejected)
            drop[i] = 2**31 - 1
            d.new[i] = 0
            pc.paged_cache_truncate(d.cdesc, drop, d.kv_len, d.held, d.table, d.free, d.num_free, d.kv_len, d.held, d.num_free, d.ws[0])
            torch.cuda.synchronize()
    assert refused and again


def test_the_step_of_the_readme():
    """The lines themselves, on a pool that two of six requests find empty, and with one that has nothing new: what these have in the cache stays."""
    from pathlib import Path
    text = (Path(__file__).parent.parent / "README.md").read_text()
    lines = [b.split("```")[0] for b in text.split("```python") if "paged_cache as pc" in b]
    assert len(lines) == 1
    g = torch.Generator().manual_seed(1)
    n, drafts, vocab, page, width, pages = 6, 3, 100, 16, 8, 40
    kv_len, new = [32, 20, 16, 48, 5, 30], [4, 4, 4, 4, 4, 0]
    held = [-(-t // page) for t in kv_len]
    table = torch.full((n, width), -1, dtype=I32)
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = torch.arange(at, at + h)
        at += h
    ints = lambda x: torch.tensor(x, dtype=I32, device="cuda")  # noqa: E731
    z = lambda *s, dtype=I32: torch.zeros(s, dtype=dtype, device="cuda")  # noqa: E731
    rows = n * (1 + drafts)
    bf16 = lambda *s: torch.randn(s, generator=g).to(BF16).cuda()  # noqa: E731
    free = torch.zeros(pages, dtype=I32)
    free[:1] = at  # one page: request 0 gets it, 2 and 3 find none
    names = dict(torch=torch, num_requests=n, max_pages=width, page_size=page, num_pages=pages, drafts=drafts, vocab=vocab, total_q=rows, new_tokens=ints(new), kv_len=ints(kv_len),
                 held=ints(held), table=table.cuda(), free_pages=free.cuda(), num_free=ints([1]), q_start=z(n + 1), slots=z(rows, dtype=I64), granted=z(n), count=z(n), k=bf16(rows, 8, 128),
                 v=bf16(rows, 8, 128), k_cache=bf16(pages, 8, page, 128), v_cache=bf16(pages, 8, page, 128), q=bf16(rows, 32, 128), o=bf16(rows, 32, 128), lse=torch.zeros((32, rows), device="cuda"),
                 target=torch.softmax(torch.randn((n, drafts + 1, vocab), generator=g), -1).cuda(), draft=torch.softmax(torch.randn((n, drafts, vocab), generator=g), -1).cuda(),
                 tokens=torch.randint(0, vocab, (n, drafts), generator=g).to(I32).cuda(), uniforms=torch.full((n, drafts), 0.99, device="cuda"), last_uniform=torch.rand(n, generator=g).cuda(),
                 accepted=z(n), rejected=z(n), out=z(n, drafts + 1))
    exec(lines[0], names)
    torch.cuda.synchronize()
    assert names["granted"].tolist() == [1, 1, 0, 0, 1, 1]
    accepted = names["accepted"].tolist()
    assert min(accepted) < drafts  # (a draft falls somewhere)
    want = [t + 1 + a if m and ok else t for t, m, a, ok in zip(kv_len, new, accepted, names["granted"].tolist())]
    assert names["kv_len"].tolist() == want and names["held"].tolist() == [-(-t // page) for t in want]
