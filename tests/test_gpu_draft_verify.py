"""Verification of drafted tokens against its definition: whole numbers, equal.  Products of a random number and a probability are exact in float64 on both sides; a running sum in float64 differs by
some 10^-15 of the total where it is taken in another order, so that a token could differ for one random number in 10^9; the tests' inputs are fixed."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc

pytestmark = pytest.mark.gpu
F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def run(target, draft, tokens, count, uniforms, last, rejected=True, stream=None):
    from paper_2509_21275_amd import draft_verify as dv
    n, places, V = target.shape
    accepted, out = torch.full((n,), -9, dtype=I32, device="cuda"), torch.full((n, places), -9, dtype=I32, device="cuda")
    rej = torch.full((n,), -9, dtype=I32, device="cuda") if rejected else None
    ws = torch.full_like(dv.alloc_workspace(n, places - 1, V), 255)
    torch.cuda.synchronize()
    dv.draft_verify(target, draft, tokens, count, uniforms, last, accepted, rej, out, ws, stream)
    torch.cuda.synchronize()
    return accepted.cpu().numpy(), None if rej is None else rej.cpu().numpy(), out.cpu().numpy()


def check(target, draft, tokens, count, uniforms, last, **kw):
    accepted, rejected, out = run(target, draft, tokens, count, uniforms, last, **kw)
    n, places, _ = target.shape
    p, q = target.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy()
    counts = np.full(n, places - 1) if count is None else np.clip(count.cpu().numpy(), 0, places - 1)
    for r in range(n):
        kept, want = orc.verify(p[r], None if q is None else q[r], tokens[r].tolist(), counts[r], uniforms[r].tolist(), float(last[r]))
        assert accepted[r] == kept and out[r].tolist() == want, (r, accepted[r], kept, out[r], want)
        assert rejected is None or rejected[r] == counts[r] - kept
    return accepted, out


def inputs(n, K, V, dtype=F32, given=True, seed=0, noise=0.7, pad=0):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn((n, K + 1, V), generator=g) * 2
    guess = torch.softmax(logits[:, :K] + noise * torch.randn((n, K, V), generator=g), -1)
    tokens = torch.multinomial(guess.reshape(-1, V), 1, generator=g).view(n, K).to(I32) if K else torch.zeros((n, 0), dtype=I32)

    def padded(x):
        y = torch.full((*x.shape[:2], V + pad), float("nan"), dtype=dtype, device="cuda")
        y[..., :V] = x.to(dtype)
        return y[..., :V]

    return (padded(torch.softmax(logits, -1)), padded(guess) if given else None, tokens.cuda(), None, torch.rand((n, K), generator=g).cuda(), torch.rand(n, generator=g).cuda())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,K,V,given,pad", [(1, 1, 1, True, 0), (1, 0, 1000, False, 0), (3, 2, 2, True, 0), (64, 4, 37, True, 0), (40, 8, 1023, True, 1), (40, 8, 1025, False, 3), (16, 5, 32000, True, 0),
                                             (7, 3, 50257, True, 8), (2, 3, 262144, True, 0), (1, 2, 300001, False, 0), (300, 64, 130, True, 0), (500, 2, 9000, True, 0)])
def test_against_the_definition(n, K, V, given, pad, dtype):
    print(n, K, V, given, pad, dtype, flush=True)
    a = inputs(n, K, V, dtype, given, seed=n + K + V, pad=pad)
    check(*a)
    if K:
        g = torch.Generator().manual_seed(1)
        check(*a[:3], torch.randint(-2, K + 3, (n,), generator=g).to(I32).cuda(), *a[4:], rejected=False)


def test_borders():
    """Probabilities and random numbers that are multiples of 1/64, so that every comparison and sum is exact: u q = p does not keep a token, and a running sum equal to the share is not past it."""
    g = torch.Generator().manual_seed(2)
    n, K, V = 400, 4, 24
    p = torch.zeros((n, K + 1, V)).scatter_add_(2, torch.randint(0, V, (n, K + 1, 64), generator=g), torch.full((n, K + 1, 64), 1 / 64))
    q = torch.zeros((n, K, V)).scatter_add_(2, torch.randint(0, V, (n, K, 64), generator=g), torch.full((n, K, 64), 1 / 64))
    q[::3] = p[::3, :K]  # as the target: nothing is left where a token falls by u = 1
    tokens = torch.randint(0, V, (n, K), generator=g).to(I32)
    u = torch.randint(0, 8, (n, K), generator=g) / 8
    u[::9] = 1.0  # (out of range: falls, as p < p does not hold, and the draft leaves nothing)
    last = torch.randint(0, 64, (n,), generator=g) / 64
    accepted, _ = check(p.cuda(), q.cuda(), tokens.cuda(), None, u.cuda(), last.cuda())
    assert len(set(accepted.tolist())) == K + 1
    check(p.cuda(), None, tokens.cuda(), None, u.cuda(), last.cuda())


def test_what_is_not_a_probability():
    """NaN, infinities, negative numbers, rows of zeros, tokens outside the vocabulary, random numbers out of [0, 1)."""
    n, K, V = 64, 3, 2500
    target, draft, tokens, _, u, last = inputs(n, K, V, seed=3)
    g = torch.Generator().manual_seed(4)
    for t in (target, draft):
        for value in (float("nan"), float("inf"), -float("inf"), -1.0):
            t.view(-1)[torch.randint(0, t.numel(), (2000,), generator=g).cuda()] = value
    target[5], target[6, :, 1:], draft[7], target[8] = 0.0, 0.0, 0.0, float("nan")
    tokens[9:14, 0] = torch.tensor([-1, V, 2**31 - 1, -2**31, V - 1], dtype=I32)
    last[20:24] = torch.tensor([1.0, 2.0, -1.0, 0.0])
    u[24:26] = torch.tensor([[float("nan")] * K, [-1.0] * K])
    check(target, draft, tokens, None, u, last)
    check(target, None, tokens, None, u, last)


def test_rows_that_do_not_matter_are_not_read():
    """All rows but the one a token is drawn from hold NaN everywhere but at the drafted tokens."""
    n, K, V = 32, 5, 3000
    target, draft, tokens, _, u, last = inputs(n, K, V, seed=5)
    accepted, out = check(target, draft, tokens, None, u, last)
    j = torch.arange(K + 1, device="cuda")
    kept = torch.tensor(accepted, device="cuda")
    for t, places in ((target, K + 1), (draft, K)):
        hide = (j[None, :places, None] != kept[:, None, None]).expand(n, places, V).clone()
        hide.scatter_(2, torch.nn.functional.pad(tokens, (0, places - K)).long()[:, :places, None], False)
        t[hide] = float("nan")
    again = run(target, draft, tokens, None, u, last)
    assert np.array_equal(again[0], accepted) and np.array_equal(again[2], out)


def test_tokens_are_distributed_as_the_target():
    """The first token of 40000 requests with the same probabilities: frequencies within 5 standard deviations (of 16 tokens, by a fixed seed) of the target's, whatever the draft proposes."""
    n, V = 40000, 16
    g = torch.Generator().manual_seed(6)
    p, q = torch.softmax(torch.randn(V, generator=g), 0), torch.softmax(torch.randn(V, generator=g), 0)
    target, draft = p.expand(n, 2, V).contiguous().cuda(), q.expand(n, 1, V).contiguous().cuda()
    tokens = torch.multinomial(q, n, replacement=True, generator=g).to(I32)[:, None].cuda()
    _, _, out = run(target, draft, tokens, None, torch.rand((n, 1), generator=g).cuda(), torch.rand(n, generator=g).cuda())
    got = np.bincount(out[:, 0], minlength=V) / n
    want = p.double().numpy()
    assert np.all(np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / n))


def test_rows_past_offsets_of_32_bits():
    """Rows more than 2^31 elements behind the first."""
    n, K, V = 20, 3, 5000
    target, draft, tokens, _, u, last = inputs(n, K, V, BF16, seed=7)
    apart = (1 << 32) // (n * (K + 1)) + 1
    far = []
    for t, m in ((target, K + 1), (draft, K)):
        x = torch.empty((n * m, apart), dtype=BF16, device="cuda")[:, :V].unflatten(0, (n, m))
        x.copy_(t)
        far.append(x)
    print("rows past 2^32 elements", flush=True)
    check(*far, tokens, None, u, last)


def test_more_rows_than_a_launch_has_workgroups_for():
    """5.6 million requests of 8193 tokens (92 GB): three workgroups to each would be more threads than a launch can have.  All weight on one token, or on two."""
    from paper_2509_21275_amd import draft_verify as dv
    n, V = (1 << 24) // 3 + 1, 8193
    if torch.cuda.mem_get_info()[0] < 130e9:
        pytest.skip("needs 130 GB")
    first = torch.randint(0, V - 1, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    second = torch.where(torch.arange(n, device="cuda") % 2 == 0, V - 1, first)
    target = torch.zeros((n, 1, V), dtype=BF16, device="cuda")
    for at in (first, second):
        target.view(-1)[torch.arange(n, device="cuda") * V + at] = 0.5
    last = torch.rand(n, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    accepted, out = torch.full((n,), -9, dtype=I32, device="cuda"), torch.full((n, 1), -9, dtype=I32, device="cuda")
    none, nothing = torch.zeros((n, 0), dtype=I32, device="cuda"), torch.zeros((n, 0), device="cuda")
    print("92 GB of probabilities", flush=True)
    dv.draft_verify(target, None, none, None, nothing, last, accepted, None, out, dv.alloc_workspace(n, 0, V))
    torch.cuda.synchronize()
    assert not accepted.any() and torch.equal(out[:, 0].long(), torch.where(last < 0.5, first, second))


def test_replayed_graph():
    from paper_2509_21275_amd import draft_verify as dv
    n, K, V = 50, 4, 20000
    sets = [inputs(n, K, V, seed=s) for s in (8, 9, 10)]
    target, draft, tokens, _, u, last = (None if t is None else t.clone() for t in sets[0])
    accepted, rejected, out = (torch.zeros(s, dtype=I32, device="cuda") for s in ((n,), (n,), (n, K + 1)))
    ws = dv.alloc_workspace(n, K, V)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dv.draft_verify(target, draft, tokens, None, u, last, accepted, rejected, out, ws)
    torch.cuda.synchronize()
    for s in sets + sets[:1]:
        for to, x in zip((target, draft, tokens, u, last), (s[0], s[1], s[2], s[4], s[5])):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        want = run(*s, stream=side)
        assert np.array_equal(accepted.cpu().numpy(), want[0]) and np.array_equal(rejected.cpu().numpy(), want[1]) and np.array_equal(out.cpu().numpy(), want[2])
        torch.ones(1000, device="cuda").sum().item()
