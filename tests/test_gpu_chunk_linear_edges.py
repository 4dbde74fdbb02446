"""Linear attention at the edges of what a call may be: gradients of states in place where no sequence is cut; outputs that are rounded to bf16 once;
decays above 1 whose powers leave float32 soon behind the last token, and decays that are no numbers.

Tolerance of outputs: half a step of bf16 for the result, 2^-8 of its value.  Before that, what is an operand of a product (weighted scores, the state, the weighted rows in the sums that become the state) is the
sum of two bf16 terms, off by at most 2^-8 * 2^-8 = 2^-16 of its value, 2^-16 / sqrt(3) in root mean square.  With the oracle's root of the sum of squares of what scores and states contribute (the sums' own
products contribute as much as the state at most, so sqrt(2) of it), six standard deviations are 6 sqrt(2) 2^-16 / sqrt(3) < 5 * 2^-16 of it.  Float32 sums: 2^-18 of the tensor's largest value."""
import pytest
import torch

from oracle import linear_oracle as orc

pytestmark = pytest.mark.gpu


def normal(shape, seed, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("d,H,Hk", [(256, 16, 16), (256, 8, 2), (128, 16, 16), (64, 4, 2)])
def test_gradients_of_states_in_place_uncut(d, H, Hk):
    """dk and dv both start from the gradient of the state behind a sequence, and its place is where the gradient of the state before it goes: with one tensor the results have the same bits as with two, also
    with more workgroups than the chip holds at once and short sequences among long ones."""
    from paper_2509_21275_amd import chunk_linear as cl
    lens = [300, 64, 1, 17] * 16
    total, segs, at = sum(lens), [], 0
    for i, n in enumerate(lens):
        segs.append((at, n, i, i))
        at += n
    desc = cl.make_desc(segs, H, Hk, d, total, len(lens), d ** -0.5)
    if d == 256 and H == 16:
        assert cl.chunk_linear_workspace_bytes(desc) == (0, 0)  # (nothing is cut)
    q, k, v, do = (normal((total, h, d), i) for i, h in enumerate((H, Hk, Hk, H)))
    lg, ws = -torch.exp2(-torch.linspace(3.0, 8.0, Hk)).cuda(), cl.alloc_workspace(desc)
    states, given = (normal((len(lens), Hk, d, d), 10 + i, torch.float32) for i in range(2))
    print(d, H, Hk, flush=True)

    def run(d_out, d_in):
        out = [torch.empty_like(t) for t in (q, k, v)]
        cl.chunk_linear_bwd(desc, q, k, v, lg, states, do, d_out, *out, d_in, ws)
        torch.cuda.synchronize()
        return [*out, d_in]

    want = run(given, torch.empty_like(given))
    both = given.clone()
    for a, b in zip(run(both, both), want):
        assert torch.equal(a, b)


def rounded_once(name, got, want, sigma):
    assert bool(torch.isfinite(got).all()), name
    over = (got.double() - want).abs() - (2.0 ** -8 * want.abs() + 5 * 2.0 ** -16 * sigma + 2.0 ** -18 * want.abs().max())
    assert float(over.max()) <= 0, (name, float(over.max()), int((over > 0).sum()), over.numel())


@pytest.mark.parametrize("lens,H,Hk,d", [([1, 33, 64, 130], 4, 2, 64), ([700], 2, 2, 64), ([200, 65], 3, 1, 96), ([100, 500], 4, 2, 128), ([1500], 2, 2, 128), ([90, 300], 2, 1, 256)])
def test_outputs_are_rounded_once(lens, H, Hk, d):
    """From states and from none, uncut and in pieces, all query heads of a key/value head."""
    from paper_2509_21275_amd import chunk_linear as cl
    total, scale = sum(lens), d ** -0.5
    segs, at = [], 0
    for i, n in enumerate(lens):
        segs.append((at, n, i if i % 2 == 0 else -1, i))
        at += n
    q, k, v, do = (normal((total, h, d), 20 + i) for i, h in enumerate((H, Hk, Hk, H)))
    lg = -torch.exp2(-torch.linspace(2.0, 9.0, Hk)).cuda()
    states, grads = normal((len(lens), Hk, d, d), 30, torch.float32, 3.0), normal((len(lens), Hk, d, d), 31, torch.float32)
    desc = cl.make_desc(segs, H, Hk, d, total, len(lens), scale)
    ws, left, first = cl.alloc_workspace(desc), torch.empty_like(states), torch.empty_like(states)
    o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
    print(lens, H, Hk, d, flush=True)
    cl.chunk_linear_fwd(desc, q, k, v, lg, states, o, left, ws)
    cl.chunk_linear_bwd(desc, q, k, v, lg, states, do, grads, dq, dk, dv, first, ws)
    torch.cuda.synchronize()
    for start, n, a, b in segs:
        r, S0, dS = slice(start, start + n), states[a] if a >= 0 else None, grads[b]
        rounded_once("o", o[r], orc.forward(q[r], k[r], v[r], lg, scale, S0)[0], orc.rounding(q[r], k[r], v[r], lg, scale, S0))
        wq, wk, wv, _, _ = orc.backward(q[r], k[r], v[r], lg, scale, do[r], S0, dS)
        rounded_once("dq", dq[r], wq, orc.rounding(do[r], v[r], k[r], lg, scale, None if S0 is None else S0.transpose(1, 2)))
        rounded_once("dk", dk[r], wk, orc.rounding(v[r], do[r], q[r], lg, scale, dS.transpose(1, 2) / scale, backwards=True))
        rounded_once("dv", dv[r], wv, orc.rounding(k[r], q[r], do[r], lg, scale, dS / scale, backwards=True))


@pytest.mark.parametrize("n,log_decay", [(1, 10.0), (5, 10.0), (8, 10.0), (9, 5.0), (10, 2.0), (24, 3.4), (33, 2.0), (40, 2.0), (63, 1.3), (64, 1.3), (65, 1.15), (150, 0.5)])
@pytest.mark.parametrize("given", [False, True])
def test_decays_far_above_one(n, log_decay, given):
    """Powers of the decay that no token needs may be past float32's largest number (exp(88.7)): what is finite by definition is right.  Every product and sum is of float32 quality or 2^-16 of a term, in sums
    of less than 2^8 terms: 2^-14 of the sum of the terms' magnitudes (the oracle's result of the magnitudes), and half a step of bf16 for the result."""
    from paper_2509_21275_amd import chunk_linear as cl
    for d, H, Hk in ((64, 2, 1), (96, 1, 1), (128, 2, 2), (256, 1, 1)):
        q, k, v, do = (normal((n, h, d), 40 + i) for i, h in enumerate((H, Hk, Hk, H)))
        lg, scale = torch.full((Hk,), log_decay, device="cuda"), d ** -0.5
        states, grads = normal((1, Hk, d, d), 45, torch.float32), normal((1, Hk, d, d), 46, torch.float32)
        desc = cl.make_desc([(0, n, 0 if given else -1, 0)], H, Hk, d, n, 1, scale)
        ws, left, first = cl.alloc_workspace(desc), torch.empty_like(states), torch.zeros_like(states)
        o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
        print(n, log_decay, given, d, flush=True)
        cl.chunk_linear_fwd(desc, q, k, v, lg, states, o, left, ws)
        cl.chunk_linear_bwd(desc, q, k, v, lg, states, do, grads if given else None, dq, dk, dv, first if given else None, ws)
        torch.cuda.synchronize()
        S0, dS = (states[0], grads[0]) if given else (None, None)
        args, sizes = (q, k, v), [t.double().abs() for t in (q, k, v)]
        want = [*orc.forward(*args, lg, scale, S0)[:2], *orc.backward(*args, lg, scale, do, S0, dS)[:4]]
        S0, dS = (None if t is None else t.double().abs() for t in (S0, dS))
        size = [*orc.forward(*sizes, lg, scale, S0)[:2], *orc.backward(*sizes, lg, scale, do.double().abs(), S0, dS)[:4]]
        got = [o, left[0], dq, dk, dv, first[0]]
        for name, g, w, z in list(zip(("o", "state", "dq", "dk", "dv", "d_state"), got, want, size))[:6 if given else 5]:
            assert bool(torch.isfinite(g).all()), name
            over = (g.double() - w).abs() - (2.0 ** -8 * w.abs() * (g.dtype == torch.bfloat16) + 2.0 ** -14 * z)
            assert float(over.max()) <= 0, (name, float(over.max()))


@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_a_decay_that_is_no_number_shows(d):
    """A NaN in log_decay: nothing of that head comes out finite, and the other heads' results have the bits that they have without it."""
    from paper_2509_21275_amd import chunk_linear as cl
    H, Hk, lens = 6, 3, [1, 30, 64, 700]
    total, scale, segs, at = sum(lens), d ** -0.5, [], 0
    for i, n in enumerate(lens):
        segs.append((at, n, i if i % 2 else -1, i))
        at += n
    q, k, v, do = (normal((total, h, d), 50 + i) for i, h in enumerate((H, Hk, Hk, H)))
    states, grads = (normal((len(lens), Hk, d, d), 55 + i, torch.float32) for i in range(2))
    desc = cl.make_desc(segs, H, Hk, d, total, len(lens), scale)
    ws, slots = cl.alloc_workspace(desc), torch.arange(len(lens), dtype=torch.int32, device="cuda")
    print(d, flush=True)

    def run(lg):
        o, dq, dk, dv, left, first, stepped = (torch.zeros_like(t) for t in (q, q, k, v, states, states, states))
        cl.chunk_linear_fwd(desc, q, k, v, lg, states, o, left, ws)
        cl.chunk_linear_bwd(desc, q, k, v, lg, states, do, grads, dq, dk, dv, first, ws)
        single = torch.zeros_like(q[:len(lens)])
        cl.chunk_linear_step(q[:len(lens)], k[:len(lens)], v[:len(lens)], lg, states, stepped, slots, single, scale)
        torch.cuda.synchronize()
        return o, dq, dk, dv, left, first[1::2], single, stepped

    lg = torch.tensor([-0.1, -0.02, -0.005], device="cuda")
    want = run(lg)
    lg[1] = float("nan")
    for got, w in zip(run(lg), want):
        n = got.shape[1] // Hk
        assert torch.equal(got[:, :n], w[:, :n]) and torch.equal(got[:, 2 * n:], w[:, 2 * n:])
        assert not bool(torch.isfinite(got[:, n:2 * n]).any())
