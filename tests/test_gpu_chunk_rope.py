"""Rotary positions of a chunk against float64.  Tolerance: a result is rounded to bf16 once (half a step, 2^-8 of the value); before that sine and cosine are off by 2 units of
float32 at most and their argument by 2 pi 2^-25, products and sums by one unit each: together below 2^-20 of |a| + |b| of the pair, times the magnitude.  What is copied is equal."""
import ctypes

import numpy as np
import pytest
import torch

import synth
from oracle import rope_oracle as orc

pytestmark = pytest.mark.gpu


def chunk(kind):
    """Segment table, rows of the keys (more than are covered)."""
    if kind == "one":
        return [(0, 1, 0, 1)], 1
    if kind == "token_behind_context":
        return [(0, 1, 5, 100001)], 100010
    if kind == "batch":  # a serving step
        ctx = [0, 7, 4095, 33, 1, 0, 12345]
        at, segs = 0, []
        for i, c in enumerate(ctx):
            segs.append((i, 1, at, c + 1))
            at += c + 3
        return segs, at
    if kind == "hybrid":
        segs = [tuple(s) for s in synth.hybrid_chunk(203, 1501, [1, 64, 2, 333])]
        return segs, segs[-1][2] + segs[-1][3] + 4
    lens = [1 + (i * 7) % 9 for i in range(500)]  # more segments than travel with one launch
    segs = [tuple(s) for s in synth.packed_chunk(lens)]
    return segs, segs[-1][2] + segs[-1][3]


def bf16(shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def close(got, want, size):
    got = got.double().cpu().numpy()
    assert np.all(np.isfinite(got))
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size), float((np.abs(got - want) - 2.0 ** -8 * np.abs(want)).max())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind,heads,kv_heads,dim,rotary", [
    ("one", 3, 1, 64, 64), ("token_behind_context", 8, 2, 128, 128), ("batch", 32, 8, 128, 128), ("hybrid", 8, 2, 128, 64), ("hybrid", 4, 4, 96, 96),
    ("hybrid", 6, 2, 256, 256), ("hybrid", 5, 1, 256, 2), ("hybrid", 4, 2, 64, 38), ("hybrid", 4, 1, 96, 94), ("many", 4, 1, 128, 32)])
def test_both_directions(kind, heads, kv_heads, dim, rotary, interleaved):
    import paper_2509_21275_amd as ca
    from paper_2509_21275_amd import chunk_rope as cr
    segs, rows = chunk(kind)
    total = segs[-1][0] + segs[-1][1]
    desc = ca.make_desc(segs, heads, kv_heads, dim, total, rows, 0.1)
    rope = cr.make_rope(rotary, 500000.0, interleaved=interleaved, magnitude=1.25)
    freq = np.array(cr.rope_frequencies(rotary, 500000.0))
    pos, key = orc.positions_and_key_rows(segs)
    print(kind, heads, kv_heads, dim, rotary, interleaved, flush=True)
    # forward from views of a fused projection
    qkv = bf16((total, heads + 2 * kv_heads, dim), 1).cuda()
    q, k = qkv[:, :heads], qkv[:, heads:heads + kv_heads]
    q_out, k_out = torch.full((total, heads, dim), float("nan"), dtype=torch.bfloat16, device="cuda"), bf16((rows, kv_heads, dim), 2).cuda()
    before, kept = k_out.clone(), qkv.clone()
    cr.chunk_rope_fwd(desc, rope, q, k, q_out, k_out)
    torch.cuda.synchronize()
    assert torch.equal(qkv, kept)
    for got, x in ((q_out, q), (k_out[key], k)):
        x = x.double().cpu().numpy()
        close(got, orc.rotate(x, pos, freq, interleaved, 1.25), orc.size(x, freq, interleaved, 1.25))
        assert np.array_equal(got[..., rotary:].double().cpu().numpy(), x[..., rotary:])
    others = np.setdiff1d(np.arange(rows), key)
    assert torch.equal(k_out[others], before[others])
    # backward into views of the projection's gradient, from bf16 and float32 dK
    for dtype in (torch.bfloat16, torch.float32):
        dq, dk = bf16((total, heads, dim), 3).cuda(), bf16((rows, kv_heads, dim), 4, dtype).cuda()
        dk[others] = float("nan")  # (rows of others are not read)
        grad = torch.full((total, heads + 2 * kv_heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        cr.chunk_rope_bwd(desc, rope, dq, dk, grad[:, :heads], grad[:, heads:heads + kv_heads])
        torch.cuda.synchronize()
        assert bool((grad[:, heads + kv_heads:] == 7.0).all())
        for got, g in ((grad[:, :heads], dq), (grad[:, heads:heads + kv_heads], dk[key])):
            g = g.double().cpu().numpy()
            close(got, orc.rotate(g, pos, freq, interleaved, 1.25, backward=True), orc.size(g, freq, interleaved, 1.25))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rotary", [(128, 128), (96, 38), (256, 254), (64, 2)])
def test_in_place_and_one_at_a_time(dim, rotary, interleaved):
    """The same bits in place, and with one tensor only; odd element offsets and strides."""
    import paper_2509_21275_amd as ca
    from paper_2509_21275_amd import chunk_rope as cr
    segs = [tuple(s) for s in synth.packed_chunk([300, 1, 77, 2000])]
    total = 2378
    desc = ca.make_desc(segs, 4, 2, dim, total, total, 0.1)
    rope = cr.make_rope(rotary, interleaved=interleaved)
    q, k = bf16((total, 4, dim), 5).cuda(), bf16((total, 2, dim), 6).cuda()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    print(dim, rotary, interleaved, flush=True)
    cr.chunk_rope_fwd(desc, rope, q, k, q_out, k_out)
    odd = torch.zeros((total, 4 * dim + 5), dtype=torch.bfloat16, device="cuda")
    shifted = odd[:, 3:3 + 4 * dim].unflatten(1, (4, dim))
    shifted.copy_(q)
    qi, ki = q.clone(), k.clone()
    cr.chunk_rope_fwd(desc, rope, qi, None, qi, None)
    cr.chunk_rope_fwd(desc, rope, None, ki, None, ki)
    cr.chunk_rope_fwd(desc, rope, shifted, None, shifted, None)
    torch.cuda.synchronize()
    assert torch.equal(qi, q_out) and torch.equal(ki, k_out) and torch.equal(shifted, q_out)
    assert bool((odd[:, :3] == 0).all()) and bool((odd[:, 3 + 4 * dim:] == 0).all())
    cr.chunk_rope_bwd(desc, rope, qi, ki, qi, ki)
    torch.cuda.synchronize()
    for got, x in ((qi, q), (ki, k)):  # back to where it came from: two roundings of 2^-8, of a pair's size
        x = x.double().cpu().numpy()
        assert np.all(np.abs(got.double().cpu().numpy() - x) <= (2.0 ** -7 + 2.0 ** -14) * orc.size(x, np.ones(rotary // 2), interleaved))


def test_far_positions():
    """Positions around 2^21: the angle's fraction of a turn is that of 64 bits."""
    import paper_2509_21275_amd as ca
    from paper_2509_21275_amd import chunk_rope as cr
    total_kv = (1 << 21) + 40
    segs = [(0, 20, 0, (1 << 21) + 20)]
    desc = ca.make_desc(segs, 2, 1, 64, 20, total_kv, 0.1)
    rope, freq = cr.make_rope(64), np.array(cr.rope_frequencies(64))
    q = bf16((20, 2, 64), 8).cuda()
    out = torch.empty_like(q)
    cr.chunk_rope_fwd(desc, rope, q, None, out, None)
    torch.cuda.synchronize()
    x = q.double().cpu().numpy()
    close(out, orc.rotate(x, orc.positions_and_key_rows(segs)[0], freq, False), orc.size(x, freq, False))


def test_more_rows_than_a_launch_takes():
    """2^26 + 77 tokens of one head (more than 2^32 bytes, several launches of one segment): rows at the ends of launches and the last ones, in place."""
    import paper_2509_21275_amd as ca
    from paper_2509_21275_amd import chunk_rope as cr
    total = (1 << 26) + 77
    desc = ca.make_desc([(0, total, 0, total)], 1, 1, 64, total, total, 0.1)
    rope, freq = cr.make_rope(64), np.array(cr.rope_frequencies(64))
    q = torch.randn((total, 1, 64), generator=torch.Generator("cuda").manual_seed(9), device="cuda", dtype=torch.bfloat16)
    some = [0, 12345, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, (1 << 26) - 1, 1 << 26, total - 1]
    x = q[some].double().cpu().numpy()
    cr.chunk_rope_fwd(desc, rope, q, None, q, None)
    torch.cuda.synchronize()
    close(q[some], orc.rotate(x, np.array(some), freq, False), orc.size(x, freq, False))


def test_on_another_stream_and_in_a_graph():
    """Queued on a side stream, and captured (with a second table whose segments fill several launches) and replayed with eager work between."""
    import paper_2509_21275_amd as ca
    from paper_2509_21275_amd import chunk_rope as cr
    segs, rows = chunk("many")
    total = segs[-1][0] + segs[-1][1]
    desc, rope = ca.make_desc(segs, 4, 2, 128, total, rows, 0.1), cr.make_rope(128)
    q, k = bf16((total, 4, 128), 9).cuda(), bf16((total, 2, 128), 10).cuda()
    want_q, want_k, q_out, k_out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)
    cr.chunk_rope_fwd(desc, rope, q, k, want_q, want_k)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    cr.chunk_rope_fwd(desc, rope, q, k, q_out, k_out, stream=side)
    side.synchronize()
    assert torch.equal(q_out, want_q) and torch.equal(k_out, want_k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cr.chunk_rope_fwd(desc, rope, q, k, q_out, k_out)
    for _ in range(3):
        q_out.zero_(), k_out.zero_()
        graph.replay()
        cr.chunk_rope_bwd(desc, rope, want_q, None, torch.empty_like(q), None)
        torch.cuda.synchronize()
        assert torch.equal(q_out, want_q) and torch.equal(k_out, want_k)


def test_a_split_chunk_equals_the_whole_sequence():
    """Rotary positions and chunk attention of a sequence cut into two slices, forward and backward, against the uncut one: O and dQ have the same inputs either way and differ as
    the attention's own slices do (its bars 2e-2 and 5e-2 of the largest value); the keys that reach the buffer are the same bits."""
    import paper_2509_21275_amd as ca
    from gpu_util import TOL_GRAD, TOL_O, rel_err
    from paper_2509_21275_amd import chunk_rope as cr
    n, cut, H, Hk, d = 700, 411, 4, 2, 128
    q, k, v, do = (bf16((n, h, d), 20 + i).cuda() for i, h in enumerate((H, Hk, Hk, H)))
    rope = cr.make_rope(d)

    def run(slices):
        kb = torch.zeros_like(k)
        o, dq, saved = torch.empty_like(q), torch.empty_like(q), []
        for a, b in slices:
            desc = ca.make_desc([(0, b - a, 0, b)], H, Hk, d, b - a, n, d ** -0.5)
            qr, lse, ws = torch.empty_like(q[a:b]), torch.empty((H, b - a), device="cuda"), ca.alloc_workspace(desc)
            cr.chunk_rope_fwd(desc, rope, q[a:b], k[a:b], qr, kb)
            ca.chunk_attn_fwd(desc, qr, kb, v, o[a:b], lse, ws)
            saved.append((a, b, desc, qr, lse, ws))
        dk, dv, dkp = torch.zeros(k.shape, device="cuda"), torch.zeros(v.shape, device="cuda"), torch.empty_like(k)
        for a, b, desc, qr, lse, ws in reversed(saved):
            dqr = torch.empty_like(qr)
            ca.chunk_attn_bwd_f32kv(desc, qr, kb, v, o[a:b], do[a:b], lse, dqr, dk, dv, True, ws)
            cr.chunk_rope_bwd(desc, rope, dqr, dk, dq[a:b], dkp[a:b])
        torch.cuda.synchronize()
        return kb, o, dq, dkp

    whole, sliced = run([(0, n)]), run([(0, cut), (cut, n)])
    assert torch.equal(whole[0], sliced[0])
    for got, want, tol in zip(sliced[1:], whole[1:], (TOL_O, TOL_GRAD, TOL_GRAD)):
        assert rel_err(got, want.double().cpu().numpy()) <= tol
