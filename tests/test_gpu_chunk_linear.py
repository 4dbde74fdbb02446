"""Linear attention with a decay for each head against float64, token by token.

Tolerances.  Outputs: the result is rounded to bf16 (half a step, 2^-8 of the value); before that each weighted score and each element of the state is rounded to bf16
once, errors that are independent, at most 2^-8 and uniform, so 2^-8 / sqrt(3) in root mean square: with the oracle's root of the sum of squares of what they are relative to, six of these standard deviations
(of some 10^6 elements one in 500 tensors would pass six by chance if the errors were normal; they are bounded and steps average 0.72 of the largest).  Float32 sums: 2^-18 of the largest
value of the tensor.  States: float32 sums of products as good as float32's, over a few thousand terms in runs of 64: 2^-18 of the sum of the terms' magnitudes; and a power of the decay
below the smallest normal float32 (2^-126; exp(-88) is) counts as 0, which loses less than 2^-126 of the product that it weights: normal deviates, |x| < 5.6, so less than 2^-126 * 32 for each
token and query head."""
import numpy as np
import pytest
import torch

from oracle import linear_oracle as orc

pytestmark = pytest.mark.gpu


def bf16(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def f32(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda()


def close(name, got, want, sigma):
    got = got.double()
    assert bool(torch.isfinite(got).all()), name
    over = (got - want).abs() - (2.0 ** -8 * want.abs() + 6 * 2.0 ** -8 / 3 ** 0.5 * sigma + 2.0 ** -18 * want.abs().max())
    assert float(over.max()) <= 0, (name, float(over.max()), int((over > 0).sum()), over.numel())


def close_state(name, got, want, size, terms=1):
    over = (got.double() - want).abs() - 2.0 ** -18 * size - 2.0 ** -126 * 32 * terms
    assert float(over.max()) <= 0, (name, float(over.max()))


def decays(Hk, kind):
    if kind == "weak":
        return -torch.exp2(-torch.linspace(3.0, 10.0, Hk)).cuda()
    if kind == "growing":
        return torch.linspace(0.02, 0.001, Hk).cuda()
    return torch.tensor([0.0, -0.7, -30.0, float("-inf"), -3.0, -0.05, -88.0, -0.001][:Hk], device="cuda")


def check(segs, H, Hk, d, kind, num_states, total, seed=0, in_place=False):
    from paper_2509_21275_amd import chunk_linear as cl
    q, k, v, do = (bf16((total, h, d), seed + i) for i, h in enumerate((H, Hk, Hk, H)))
    lg, scale = decays(Hk, kind), d ** -0.5
    desc = cl.make_desc(segs, H, Hk, d, total, num_states, scale)
    ws = cl.alloc_workspace(desc)
    s_in = f32((num_states, Hk, d, d), seed + 5, 3.0)
    s_out = s_in.clone() if in_place else torch.full_like(s_in, 7.0)
    given = s_in.clone()
    o = torch.full((total, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    cl.chunk_linear_fwd(desc, q, k, v, lg, s_out if in_place else s_in, o, s_out, ws)
    d_out, d_in = f32((num_states, Hk, d, d), seed + 6), torch.full_like(s_in, 7.0)
    d_given = d_out.clone()
    if in_place:
        d_in = d_out
    dq, dk, dv = (torch.full((total, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for h in (H, Hk, Hk))
    cl.chunk_linear_bwd(desc, q, k, v, lg, given, do, d_out, dq, dk, dv, d_in, ws)
    torch.cuda.synchronize()
    covered, left, started = torch.zeros(total, dtype=torch.bool), set(), set()
    for start, n, a, b in segs:
        r = slice(start, start + n)
        covered[r] = True
        S0, dS = given[a] if a >= 0 else None, d_given[b] if b >= 0 else None
        want, S, size = orc.forward(q[r], k[r], v[r], lg, scale, S0)
        close("o", o[r], want, orc.rounding(q[r], k[r], v[r], lg, scale, S0))
        if b >= 0:
            close_state("state", s_out[b], S, size, n * (H // Hk))
            left.add(b)
        wq, wk, wv, dS0, size = orc.backward(q[r], k[r], v[r], lg, scale, do[r], S0, dS)
        close("dq", dq[r], wq, orc.rounding(do[r], v[r], k[r], lg, scale, None if S0 is None else S0.transpose(1, 2)))
        close("dk", dk[r], wk, orc.rounding(v[r], do[r], q[r], lg, scale, None if dS is None else dS.transpose(1, 2) / scale, backwards=True))
        close("dv", dv[r], wv, orc.rounding(k[r], q[r], do[r], lg, scale, None if dS is None else dS / scale, backwards=True))
        if a >= 0:
            close_state("d_state", d_in[a], dS0, size, n * (H // Hk))
            started.add(a)
    # what belongs to no segment stays
    for t in (o, dq, dk, dv):
        assert bool((t[~covered] == 7.0).all())
    for i in range(num_states):
        if i not in left:
            assert torch.equal(s_out[i], given[i]) if in_place else bool((s_out[i] == 7.0).all())
        if i not in started:
            assert torch.equal(d_in[i], d_given[i]) if in_place else bool((d_in[i] == 7.0).all())


def packed(lens, gap=0, states=True):
    segs, at = [], gap
    for i, n in enumerate(lens):
        segs.append((at, n, 2 * i if states and i % 2 == 0 else -1, 2 * i + 1 if states and i % 3 != 2 else -1))
        at += n + gap
    return segs, at, 2 * len(lens) + 1


@pytest.mark.parametrize("kind", ["weak", "any"])
@pytest.mark.parametrize("lens,H,Hk,d", [
    ([1], 1, 1, 64), ([1, 2, 63, 64, 65], 4, 2, 64), ([127, 128, 129, 31, 32, 33], 2, 2, 128), ([300, 5], 8, 2, 128), ([257, 100], 3, 3, 96), ([130, 1, 64], 4, 1, 256),
    ([1100], 4, 4, 64), ([513, 700], 8, 8, 128), ([1500], 2, 1, 96), ([777], 2, 2, 256), ([600], 16, 2, 128), ([90, 290], 10, 2, 64)])
def test_sequences(lens, H, Hk, d, kind):
    """Sequences around the block of 64 rows and of several pieces, packed with gaps, from given states and from none."""
    segs, total, slots = packed(lens, gap=3)
    print(lens, H, Hk, d, kind, flush=True)
    check(segs, H, Hk, d, kind, slots, total)


def test_states_in_place():
    """One tensor for the states before and behind, and one for their gradients; also where a sequence is cut into pieces."""
    for lens, H, Hk, d in (([70, 1200, 1], 2, 2, 64), ([900, 64], 4, 2, 128)):
        segs, at = [], 0
        for i, n in enumerate(lens):
            segs.append((at, n, i, i))
            at += n
        print(lens, H, Hk, d, flush=True)
        check(segs, H, Hk, d, "weak", len(lens) + 1, at, in_place=True)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,H,Hk,d", [([640, 3], 3, 1, 64), ([2500], 2, 2, 64), ([400, 129], 2, 1, 96), ([1500], 2, 2, 96), ([300, 200], 2, 2, 128), ([700], 2, 1, 128), ([500], 1, 1, 256)])
def test_pieces_and_states(lens, H, Hk, d, in_place):
    """Few and many pieces of a sequence (sums added up by the walks, or before them), each sequence from a state and to one."""
    segs, at = [], 0
    for i, n in enumerate(lens):
        segs.append((at, n, i, i if in_place else len(lens) - i))
        at += n
    print(lens, H, Hk, d, in_place, flush=True)
    check(segs, H, Hk, d, "weak", len(lens) + 1, at, seed=7, in_place=in_place)


def test_states_that_grow():
    """Decays above 1 are taken as they are."""
    for lens, H, Hk, d in (([70, 500, 1], 4, 2, 64), ([330], 2, 2, 128), ([200], 1, 1, 256)):
        segs, total, slots = packed(lens, gap=2)
        print(lens, H, Hk, d, flush=True)
        check(segs, H, Hk, d, "growing", slots, total, seed=11)


def test_many_sequences():
    """More segments than travel with one launch, some of them cut."""
    lens = [1 + (i * 37) % 90 for i in range(300)]
    lens[150] = 700
    segs, at = [], 0
    for i, n in enumerate(lens):
        segs.append((at, n, -1, i if i % 50 == 0 else -1))
        at += n
    check(segs, 2, 2, 64, "weak", 300, at)


def test_many_heads_and_sequences():
    """More pairs of a segment and a head than 2^16, one of the sequences cut; some of the heads against the oracle."""
    from paper_2509_21275_amd import chunk_linear as cl
    n, more, H, d = 24576, 127, 513, 64
    total, scale, some = n + more, d ** -0.5, [0, 255, 512]
    generator = torch.Generator("cuda").manual_seed(3)
    q, k, v = (torch.randn((total, H, d), generator=generator, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    o, lg = torch.empty_like(q), torch.full((H,), -0.002, device="cuda")
    states = torch.full((2, H, d, d), 7.0, device="cuda")
    states[0].zero_()
    desc = cl.make_desc([(0, n, 0, 0)] + [(n + i, 1, -1, 1 if i == 9 else -1) for i in range(more)], H, H, d, total, 2, scale)
    assert cl.chunk_linear_workspace_bytes(desc)[0] > 0  # (it is cut)
    cl.chunk_linear_fwd(desc, q, k, v, lg, states, o, states, cl.alloc_workspace(desc))
    torch.cuda.synchronize()
    q, k, v, o, lg, states = q[:, some], k[:, some], v[:, some], o[:, some], lg[some], states[:, some]
    want, S, size = orc.forward(q[:n], k[:n], v[:n], lg, scale)
    close("o", o[:n], want, orc.rounding(q[:n], k[:n], v[:n], lg, scale))
    close_state("state", states[0], S, size, n)
    for i in range(n, total):
        r = slice(i, i + 1)
        want, S, size = orc.forward(q[r], k[r], v[r], lg, scale)
        close("o", o[r], want, orc.rounding(q[r], k[r], v[r], lg, scale))
        if i == n + 9:
            close_state("state", states[1], S, size)


def test_scale_of_no_normal_inverse():
    """A scale whose inverse is not finite in float32: the gradients of what only the states carry are as they are with any other.  (What the scale multiplies is 2^-120 and less.)"""
    from paper_2509_21275_amd import chunk_linear as cl
    for n, d in ((100, 64), (1500, 128)):
        H, scale = 2, 2.0 ** -130
        q, k, v, do = (bf16((n, H, d), 30 + i) for i in range(4))
        lg, ds = torch.full((H,), -0.004, device="cuda"), f32((1, H, d, d), 35)
        desc = cl.make_desc([(0, n, -1, 0)], H, H, d, n, 1, scale)
        dq, dk, dv = (torch.empty_like(q) for _ in range(3))
        print(n, d, flush=True)
        cl.chunk_linear_bwd(desc, q, k, v, lg, None, do, ds, dq, dk, dv, None, cl.alloc_workspace(desc))
        torch.cuda.synchronize()
        none = torch.zeros_like(q)
        _, wk, wv, _, _ = orc.backward(q, k, v, lg, scale, do, None, ds[0])
        assert float(dq.abs().max()) < 2.0 ** -100
        close("dk", dk, wk, orc.rounding(v, none, none, lg, 1.0, ds[0].transpose(1, 2), backwards=True))
        close("dv", dv, wv, orc.rounding(k, none, none, lg, 1.0, ds[0], backwards=True))


def test_rows_past_4_gib():
    """A short sequence at the end of tensors of more than 2^32 bytes."""
    from paper_2509_21275_amd import chunk_linear as cl
    total, H, d, n = 132000, 64, 256, 100
    q, k, v, o = (torch.empty((total, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    for i, t in enumerate((q, k, v)):
        t[-n:] = bf16((n, H, d), i)
    lg = decays(8, "weak").repeat(8)
    desc = cl.make_desc([(total - n, n, -1, -1)], H, H, d, total, 0, d ** -0.5)
    cl.chunk_linear_fwd(desc, q, k, v, lg, None, o, None, cl.alloc_workspace(desc))
    torch.cuda.synchronize()
    want, _, _ = orc.forward(q[-n:], k[-n:], v[-n:], lg, d ** -0.5)
    close("o", o[-n:], want, orc.rounding(q[-n:], k[-n:], v[-n:], lg, d ** -0.5))


def test_same_bits_on_streams_and_in_graphs():
    """A forward and a backward of a chunk with cut sequences: on a side stream, captured and replayed with eager work between, always the same bits."""
    from paper_2509_21275_amd import chunk_linear as cl
    segs, total, slots = packed([1300, 20, 400])
    H, Hk, d = 4, 2, 128
    q, k, v, do = (bf16((total, h, d), 40 + i) for i, h in enumerate((H, Hk, Hk, H)))
    lg = decays(Hk, "weak")
    desc = cl.make_desc(segs, H, Hk, d, total, slots, 0.1)
    ws, s_in, ds_out = cl.alloc_workspace(desc), f32((slots, Hk, d, d), 45), f32((slots, Hk, d, d), 46)

    def outputs():
        return [torch.zeros_like(q), torch.zeros_like(s_in), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(s_in)]

    def both(out, stream=None):
        cl.chunk_linear_fwd(desc, q, k, v, lg, s_in, out[0], out[1], ws, stream=stream)
        cl.chunk_linear_bwd(desc, q, k, v, lg, s_in, do, ds_out, *out[2:], ws, stream=stream)

    want, out, side, graph = outputs(), outputs(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    both(want)
    torch.cuda.synchronize()
    both(out, side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    with torch.cuda.graph(graph, stream=side):
        both(out)
    for _ in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        both(outputs())
        torch.cuda.synchronize()


def test_values_that_are_not_finite_stay_in_their_sequence():
    from paper_2509_21275_amd import chunk_linear as cl
    lens, H, d = [200, 70, 130], 2, 64
    segs = [(0, 200, -1, -1), (200, 70, -1, -1), (270, 130, -1, -1)]
    q, k, v, do = (bf16((400, H, d), 50 + i) for i in range(4))
    desc = cl.make_desc(segs, H, H, d, 400, 0, 0.1)
    lg, ws = decays(H, "weak"), cl.alloc_workspace(desc)

    def run():
        out = [torch.empty_like(q) for _ in range(4)]
        cl.chunk_linear_fwd(desc, q, k, v, lg, None, out[0], None, ws)
        cl.chunk_linear_bwd(desc, q, k, v, lg, None, do, None, *out[1:], None, ws)
        torch.cuda.synchronize()
        return out

    want = run()
    k[230] = float("nan")
    v[240, 0, 3] = float("inf")
    do[250] = float("nan")
    for got, w in zip(run(), want):
        assert torch.equal(got[:200], w[:200]) and torch.equal(got[270:], w[270:])
        assert not bool(torch.isfinite(got[200:270]).all())


def test_slices_equal_the_whole_sequence():
    """A sequence in slices, states carried forward and their gradients back, against the uncut one: both within the tolerance of the same float64 values."""
    from paper_2509_21275_amd import chunk_linear as cl
    n, H, Hk, d = 1000, 4, 2, 128
    q, k, v, do = (bf16((n, h, d), 60 + i) for i, h in enumerate((H, Hk, Hk, H)))
    lg, scale = decays(Hk, "weak"), d ** -0.5
    want, S, size = orc.forward(q, k, v, lg, scale)
    wants = orc.backward(q, k, v, lg, scale, do)
    for cuts in ([0, 1000], [0, 333, 334, 900, 1000], [0, 64, 1000]):
        o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
        states = torch.zeros((len(cuts), Hk, d, d), device="cuda")
        pieces = []
        for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
            desc = cl.make_desc([(0, b - a, i, i + 1)], H, Hk, d, b - a, len(cuts), scale)
            pieces.append((slice(a, b), desc, cl.alloc_workspace(desc)))
            cl.chunk_linear_fwd(desc, q[a:b], k[a:b], v[a:b], lg, states, o[a:b], states, pieces[-1][2])
        grads = torch.zeros_like(states)
        for r, desc, ws in reversed(pieces):
            cl.chunk_linear_bwd(desc, q[r], k[r], v[r], lg, states, do[r], grads, dq[r], dk[r], dv[r], grads, ws)
        torch.cuda.synchronize()
        print(cuts, flush=True)
        # What is rounded follows from the slices: blocks begin at a slice's first row, with the exact state before (behind) the slice.
        before, behind = [None], [None]
        for a, b in zip(cuts, cuts[1:]):
            before.append(orc.forward(q[a:b], k[a:b], v[a:b], lg, scale, before[-1])[1])
        for a, b in reversed(list(zip(cuts, cuts[1:]))):
            behind.append(orc.backward(q[a:b], k[a:b], v[a:b], lg, scale, do[a:b], None, behind[-1])[3])
        behind = behind[-2::-1]
        for (a, b), S0, dS in zip(zip(cuts, cuts[1:]), before, behind):
            r = slice(a, b)
            close("o", o[r], want[r], orc.rounding(q[r], k[r], v[r], lg, scale, S0))
            close("dq", dq[r], wants[0][r], orc.rounding(do[r], v[r], k[r], lg, scale, None if S0 is None else S0.transpose(1, 2)))
            close("dk", dk[r], wants[1][r], orc.rounding(v[r], do[r], q[r], lg, scale, None if dS is None else dS.transpose(1, 2) / scale, backwards=True))
            close("dv", dv[r], wants[2][r], orc.rounding(k[r], q[r], do[r], lg, scale, None if dS is None else dS / scale, backwards=True))
        close_state("state", states[-1], S, size)
        close_state("d_state", grads[0], wants[3], wants[4])


@pytest.mark.parametrize("B,H,Hk,d", [(1, 1, 1, 64), (5, 4, 2, 128), (9, 16, 2, 64), (3, 6, 6, 96), (4, 5, 1, 256), (300, 2, 1, 64)])
@pytest.mark.parametrize("kind", ["weak", "any"])
def test_step(B, H, Hk, d, kind):
    """One token of each of a batch; rows of a padded batch (no slot) and slots of others stay; several tokens of a sequence in the order of the rows; in place and not."""
    from paper_2509_21275_amd import chunk_linear as cl
    slots = torch.randperm(B + 3, generator=torch.Generator().manual_seed(B)).to(torch.int32)[:B]
    if B > 3:
        slots[1], slots[3] = -1, slots[0]
    if B > 8:
        slots[5], slots[6], slots[7] = slots[0], B + 3, 1 << 30
    q, k, v = (bf16((B, h, d), 70 + i) for i, h in enumerate((H, Hk, Hk)))
    lg, scale, before = decays(Hk, kind), d ** -0.5, f32((B + 3, Hk, d, d), 75, 3.0)
    print(B, H, Hk, d, kind, flush=True)
    results = []
    for in_place in (False, True):
        src = before.clone()
        dst = src if in_place else torch.full_like(before, 7.0)
        o = torch.full((B, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
        cl.chunk_linear_step(q, k, v, lg, src, dst, slots.cuda(), o, scale)
        torch.cuda.synchronize()
        results.append((o, dst))
    assert torch.equal(results[0][0], results[1][0])
    o, dst = results[0]
    rows = {}
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < B + 3:
            rows.setdefault(s, []).append(i)
        else:
            assert bool((o[i] == 7.0).all())
    for s in range(B + 3):
        if s not in rows:
            assert bool((dst[s] == 7.0).all()) and torch.equal(results[1][1][s], before[s])
            continue
        r = rows[s]
        want, S, size = orc.forward(q[r], k[r], v[r], lg, scale, before[s])
        assert torch.equal(dst[s], results[1][1][s])
        close_state("state", dst[s], S, size, len(r))  # (nothing is rounded to bf16 but the result)
        close("o", o[r], want, torch.zeros_like(want))


def test_step_continues_a_forward():
    """A prompt, then single tokens, captured in a graph, against the whole sequence."""
    from paper_2509_21275_amd import chunk_linear as cl
    n, m, H, Hk, d = 150, 6, 4, 2, 128
    q, k, v = (bf16((n + m, h, d), 80 + i) for i, h in enumerate((H, Hk, Hk)))
    lg, scale = decays(Hk, "weak"), d ** -0.5
    states = torch.zeros((3, Hk, d, d), device="cuda")
    desc = cl.make_desc([(0, n, -1, 1)], H, Hk, d, n, 3, scale)
    o = torch.empty_like(q)
    cl.chunk_linear_fwd(desc, q[:n], k[:n], v[:n], lg, None, o[:n], states, cl.alloc_workspace(desc))
    slot = torch.tensor([1], dtype=torch.int32, device="cuda")
    qt, kt, vt, ot = (torch.zeros_like(t[:1]) for t in (q, k, v, q))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cl.chunk_linear_step(qt, kt, vt, lg, states, states, slot, ot, scale)
    for t in range(n, n + m):
        for to, x in ((qt, q), (kt, k), (vt, v)):
            to.copy_(x[t:t + 1])
        graph.replay()
        o[t:t + 1].copy_(ot)
    torch.cuda.synchronize()
    want, S, size = orc.forward(q, k, v, lg, scale)
    close("o", o, want, orc.rounding(q, k, v, lg, scale))
    close_state("state", states[1], S, size)


def test_gradients_against_differences():
    """The kernel's gradients against central differences of the oracle's forward along random directions.  The kernel's carry independent roundings of some 2^-8
    each (three of them): over a direction's terms their root sum of squares, times four."""
    from paper_2509_21275_amd import chunk_linear as cl
    n, H, Hk, d = 80, 2, 1, 64
    q, k, v, do = (bf16((n, h, d), 90 + i) for i, h in enumerate((H, Hk, Hk, H)))
    lg, scale = torch.tensor([-0.05], device="cuda"), d ** -0.5
    s0, ds = f32((2, Hk, d, d), 95), f32((2, Hk, d, d), 96)
    desc = cl.make_desc([(0, n, 0, 1)], H, Hk, d, n, 2, scale)
    dq, dk, dv, d0 = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.zeros_like(s0)
    cl.chunk_linear_bwd(desc, q, k, v, lg, s0, do, ds, dq, dk, dv, d0, cl.alloc_workspace(desc))
    torch.cuda.synchronize()
    args = [q.double(), k.double(), v.double(), s0[0].double()]

    def loss(a):
        o, S, _ = orc.forward(*a[:3], lg, scale, a[3])
        return float((o * do.double()).sum() + (S * ds[1].double()).sum())

    for i, g in enumerate((dq, dk, dv, d0[0])):
        way = torch.randn(args[i].shape, generator=torch.Generator().manual_seed(i), dtype=torch.float64).cuda()
        up, down = ([a + (s * 1e-4 * way if j == i else 0) for j, a in enumerate(args)] for s in (1, -1))
        slope = (loss(up) - loss(down)) / 2e-4
        terms = g.double() * way
        assert abs(slope - float(terms.sum())) <= 4 * 3 ** 0.5 * 2.0 ** -8 * float((terms ** 2).sum()) ** 0.5 + 1e-6 * abs(slope), i
