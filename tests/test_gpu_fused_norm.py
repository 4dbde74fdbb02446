"""Norms around a block against float64.  Tolerance: bf16 results are rounded once (half a step, 2^-8 of the value); float32 rounding before that: a few dozen operations and sums of
cols (rows) terms in trees and short runs, below 2^-18 of the magnitudes of the terms a result is formed from (the oracle's sizes; 64 units of float32)."""
import numpy as np
import pytest
import torch

from oracle import norm_oracle as orc

pytestmark = pytest.mark.gpu
ALL = dict(y=True, gate=True, residual=True, post=True, pre=True)


def make(rows, cols, seed, dtype=torch.bfloat16, scale=1.0, pad=0):
    t = torch.randn((rows, cols + pad), generator=torch.Generator().manual_seed(seed)) * scale
    return t.to(dtype).cuda()[:, :cols]


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def close(name, got, want, size):
    got = wide(got)
    half_step = 2.0 ** -8 if name not in ("f32",) else 0.0
    assert np.all(np.isfinite(got)), name
    over = np.abs(got - want) - half_step * np.abs(want) - 2.0 ** -18 * size
    assert np.all(over <= 0), (name, float(over.max()))


def case(rows, cols, parts, kind, rtype, wtype, pad, seed):
    p = {**ALL, **parts}
    y = make(rows, cols, seed, scale=0.7, pad=pad) if p["y"] else None
    gate = make(rows, cols, seed + 1, pad=pad, scale=2.0) if p["gate"] else None
    residual = make(rows, cols, seed + 2, rtype, 2.0, pad) if p["residual"] else None
    post = (1 + 0.3 * make(1, cols, seed + 3, torch.float32)[0]).to(wtype) if p["post"] else None
    pre = (1 + 0.3 * make(1, cols, seed + 4, torch.float32)[0]).to(wtype) if p["pre"] else None
    return y, gate, residual, post, pre


SHAPES = [(1, 1), (3, 7), (5, 8), (33, 96), (70, 128), (17, 129), (40, 256), (9, 500), (8, 512), (6, 1001), (5, 1024), (4, 2048), (3, 2049), (300, 4096), (3, 4095),
          (5, 8192), (2, 8200), (3, 16384), (2, 16383), (2500, 64), (700, 1024)]
KINDS = ["sigmoid", "silu", "plain"]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("rtype", [torch.bfloat16, torch.float32])
def test_sizes(rows, cols, rtype):
    """Every length of row around the steps between thread counts, with every part, padded (odd strides) or not; forward and backward."""
    from paper_2509_21275_amd import fused_norm as fn
    kind, wtype, pad = KINDS[cols % 3], (torch.float32, torch.bfloat16)[rows % 2], (0, 3, 8)[(rows + cols) % 3]
    print(rows, cols, rtype, kind, wtype, pad, flush=True)
    run(fn, rows, cols, {}, kind, rtype, wtype, pad)


@pytest.mark.parametrize("cols", [80, 1024, 3000, 8192])
@pytest.mark.parametrize("parts", [
    dict(gate=False), dict(residual=False), dict(residual=False, pre=False), dict(post=False), dict(pre=False), dict(gate=False, post=False), dict(gate=False, post=False, pre=False),
    dict(y=False, gate=False, post=False)])
def test_parts_left_out(cols, parts):
    from paper_2509_21275_amd import fused_norm as fn
    print(cols, parts, flush=True)
    run(fn, 37, cols, parts, "silu", (torch.bfloat16, torch.float32)[cols % 3 % 2], torch.bfloat16, 0)


def run(fn, rows, cols, parts, kind, rtype, wtype, pad, eps=1e-5, alpha=0.75, beta=0.5):
    y, gate, residual, post, pre = case(rows, cols, parts, kind, rtype, wtype, pad, rows * 31 + cols)
    if residual is None:
        rtype = torch.bfloat16
    out = torch.full((rows, cols + pad), 9.0, dtype=rtype, device="cuda")
    h = torch.full((rows, cols + pad), 9.0, dtype=torch.bfloat16, device="cuda") if pre is not None else None
    opts = dict(eps=eps, gate_kind=kind, residual_scale=alpha, block_scale=beta)
    fn.fused_norm_fwd(y, gate, residual, post, pre, out[:, :cols], None if h is None else h[:, :cols], **opts)
    torch.cuda.synchronize()
    want, sizes = orc.forward(*map(wide, (y, gate, residual, post, pre)), eps, kind, alpha, beta)
    close("f32" if rtype == torch.float32 else "out", out[:, :cols], want["out"], sizes["out"])
    if h is not None:
        close("h", h[:, :cols], want["h"], sizes["h"])
    assert bool((out[:, cols:] == 9.0).all()) and (h is None or bool((h[:, cols:] == 9.0).all()))
    # backward at the stored sum
    stored = out[:, :cols]
    d_out, d_h = make(rows, cols, 5, rtype, pad=pad), make(rows, cols, 6, pad=pad) if pre is not None else None
    dy, dg = (torch.full((rows, cols + pad), 9.0, dtype=torch.bfloat16, device="cuda")[:, :cols] if t is not None else None for t in (y, gate))
    dr = torch.full((rows, cols), 9.0, dtype=rtype, device="cuda")
    dpost, dpre = (torch.full((cols,), float("nan"), device="cuda") if t is not None else None for t in (post, pre))
    ws = fn.alloc_workspace(rows, cols)
    fn.fused_norm_bwd(y, gate, stored, post, pre, d_out, d_h, dy, dg, dr, dpost, dpre, ws, **opts)
    torch.cuda.synchronize()
    want, sizes = orc.backward(*map(wide, (y, gate, stored, post, pre, d_out, d_h)), eps, kind, alpha, beta)
    got = {"dy": dy, "d_gate": dg, "d_residual": dr, "d_post": dpost, "d_pre": dpre}
    for name in want:
        f32 = name in ("d_post", "d_pre") or (name == "d_residual" and rtype == torch.float32)
        close("f32" if f32 else name, got[name], want[name], sizes[name])
    # gradients of weights are added to, with the same sums; without them, and without the residual's, the others are the same bits
    if post is not None or pre is not None:
        more = [None if t is None else torch.full_like(t, 2.0) for t in (dpost, dpre)]
        fn.fused_norm_bwd(y, gate, stored, post, pre, d_out, d_h, None, None, None, *more, ws, accumulate_weights=True, **opts)
        torch.cuda.synchronize()
        assert all(t is None or torch.equal(t, w + 2.0) for t, w in zip(more, (dpost, dpre)))
    if y is not None:
        dy2 = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
        fn.fused_norm_bwd(y, gate, stored, post, pre, d_out, d_h, dy2, None, None, None, None, None, **opts)
        torch.cuda.synchronize()
        assert torch.equal(dy2, dy)


def test_gradients_against_differences():
    """The gradients that the kernel gives against central differences of the oracle's forward along random directions: independent of the oracle's gradient
    formulas.  The kernel's dy, d_gate and d_residual carry bf16 roundings of random sign: of 2 * 96 products each, sqrt(192) * 2^-9 of a product's size, against sums of sqrt(192) products' size."""
    from paper_2509_21275_amd import fused_norm as fn
    rows, cols, eps, kind, alpha, beta = 2, 96, 1e-3, "silu", 0.75, 0.5
    y, gate, residual, post, pre = case(rows, cols, {}, kind, torch.float32, torch.float32, 0, 77)
    out, h = torch.empty_like(residual), torch.empty_like(y)
    opts = dict(eps=eps, gate_kind=kind, residual_scale=alpha, block_scale=beta)
    fn.fused_norm_fwd(y, gate, residual, post, pre, out, h, **opts)
    d_out, d_h = make(rows, cols, 5, torch.float32), make(rows, cols, 6)
    dy, dg, dr = torch.empty_like(y), torch.empty_like(gate), torch.empty_like(residual)
    dpost, dpre = torch.empty_like(post), torch.empty_like(pre)
    fn.fused_norm_bwd(y, gate, out, post, pre, d_out, d_h, dy, dg, dr, dpost, dpre, fn.alloc_workspace(rows, cols), **opts)
    torch.cuda.synchronize()
    args = [wide(t) for t in (y, gate, residual, post, pre)]

    def loss(a):
        o, _ = orc.forward(*a, eps, kind, alpha, beta)
        return float((o["out"] * wide(d_out)).sum() + (o["h"] * wide(d_h)).sum())

    rng = np.random.default_rng(3)
    for i, g in enumerate((dy, dg, dr, dpost, dpre)):
        way = rng.standard_normal(args[i].shape)
        step = 1e-5
        up, down = ([a + (s * step * way if j == i else 0) for j, a in enumerate(args)] for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * step)
        terms = wide(g) * way
        assert abs(slope - terms.sum()) <= 2.0 ** -8 * 4 * np.sqrt((terms ** 2).sum()) + 1e-6, i


def test_in_place_streams_and_graphs():
    """Outputs over inputs, a side stream, and a captured forward and backward replayed with eager work between, give the same bits."""
    from paper_2509_21275_amd import fused_norm as fn
    rows, cols = 1500, 4096
    y, gate, residual, post, pre = case(rows, cols, {}, "silu", torch.bfloat16, torch.bfloat16, 0, 5)
    out, h, ws = torch.empty_like(residual), torch.empty_like(y), fn.alloc_workspace(rows, cols)
    d_out, d_h = make(rows, cols, 6), make(rows, cols, 7)
    grads = [torch.empty_like(y), torch.empty_like(y), torch.empty_like(y), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]

    def both(res, out, h, d_out, d_h, grads, stream=None):
        fn.fused_norm_fwd(y_, gate_, res, post, pre, out, h, gate_kind="silu", stream=stream)
        fn.fused_norm_bwd(y_, gate_, out, post, pre, d_out, d_h, *grads, ws, gate_kind="silu", stream=stream)

    y_, gate_ = y, gate
    both(residual, out, h, d_out, d_h, grads)
    torch.cuda.synchronize()
    y_, gate_, r2, do2, dh2 = (t.clone() for t in (y, gate, residual, d_out, d_h))
    g2 = [y_, gate_, do2, torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")]
    both(r2, r2, torch.empty_like(h), do2, dh2, g2)
    torch.cuda.synchronize()
    assert torch.equal(r2, out) and all(torch.equal(a, b) for a, b in zip(g2, grads))
    y_, gate_ = y, gate
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    out2, h2, g2 = torch.empty_like(out), torch.empty_like(h), [torch.empty_like(g) for g in grads]
    both(residual, out2, h2, d_out, d_h, g2, stream=side)
    side.synchronize()
    assert torch.equal(out2, out) and torch.equal(h2, h) and all(torch.equal(a, b) for a, b in zip(g2, grads))
    with torch.cuda.graph(graph, stream=side):
        both(residual, out2, h2, d_out, d_h, g2)
    for _ in range(3):
        for t in (out2, h2, *g2):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, out) and torch.equal(h2, h) and all(torch.equal(a, b) for a, b in zip(g2, grads))
        both(residual, torch.empty_like(out), torch.empty_like(h), d_out, d_h, [torch.empty_like(g) for g in grads])  # (eager, on the current stream)
        torch.cuda.synchronize()


def test_no_rows_zero_rows_and_values_that_are_not_numbers():
    """No rows: gradients of weights are 0, or stay when added to.  A row of zeros has a finite norm; a NaN or an infinity stays in its row, but for the weights' gradients."""
    from paper_2509_21275_amd import fused_norm as fn
    empty = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w, dw = torch.ones(64, device="cuda"), [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    fn.fused_norm_fwd(empty, None, empty, w, w, empty, empty)
    fn.fused_norm_bwd(empty, None, empty, w, w, empty, empty, empty, None, empty, *dw, fn.alloc_workspace(0, 64), accumulate_weights=True)
    torch.cuda.synchronize()
    assert all(bool((t == 3.0).all()) for t in dw)
    fn.fused_norm_bwd(empty, None, empty, w, w, empty, empty, empty, None, empty, *dw, fn.alloc_workspace(0, 64))
    torch.cuda.synchronize()
    assert all(bool((t == 0.0).all()) for t in dw)
    for cols in (100, 1000, 5000):
        rows = 12
        y, gate, residual, post, pre = case(rows, cols, {}, "sigmoid", torch.bfloat16, torch.float32, 0, 9)
        clean = [t.clone() for t in (y, residual)]
        y[3] = 0
        residual[3] = 0
        y[5, cols - 1] = float("nan")
        residual[7, 1] = float("inf")

        def fwd_bwd(y, residual):
            out, h = torch.empty_like(residual), torch.empty_like(y)
            fn.fused_norm_fwd(y, gate, residual, post, pre, out, h)
            g = [torch.empty_like(y) for _ in range(3)]
            fn.fused_norm_bwd(y, gate, out, post, pre, out, h, *g, None, None, None)
            torch.cuda.synchronize()
            return [out, h, *g]

        got, want = fwd_bwd(y, residual), fwd_bwd(*clean)
        keep = [r for r in range(rows) if r not in (3, 5, 7)]
        assert all(torch.equal(a[keep], b[keep]) for a, b in zip(got, want))
        assert all(bool(torch.isfinite(t[3]).all()) for t in got) and all(bool((t[3] == 0).all()) for t in got[:2])
        assert bool(torch.isnan(got[0][5]).all()) and bool(torch.isnan(got[1][5]).all())


@pytest.mark.parametrize("cols", [80, 256, 1024, 8192, 16384])
@pytest.mark.parametrize("wtype", [torch.bfloat16, torch.float32])
def test_weights_at_any_address(cols, wtype):
    """Weights that begin one element behind an aligned address (a row of a stacked parameter), and their gradients too: the bits of aligned ones."""
    from paper_2509_21275_amd import fused_norm as fn
    rows = 9
    y, gate, residual, post, pre = case(rows, cols, {}, "silu", torch.bfloat16, wtype, 0, cols)
    d_out, d_h, ws = make(rows, cols, 6), make(rows, cols, 7), fn.alloc_workspace(rows, cols)
    results = []
    for shift in (0, 1):
        w = [torch.cat([t.new_full((shift,), float("nan")), t])[shift:] for t in (post, pre)]
        assert all(t.data_ptr() % 16 == shift * t.element_size() for t in w)
        out, h, dy, dg, dr = (torch.empty_like(y) for _ in range(5))
        dw = [torch.full((cols + shift,), 7.0, device="cuda")[shift:] for _ in range(2)]
        print(cols, wtype, shift, flush=True)
        fn.fused_norm_fwd(y, gate, residual, *w, out, h, gate_kind="silu")
        fn.fused_norm_bwd(y, gate, out, *w, d_out, d_h, dy, dg, dr, *dw, ws, gate_kind="silu")
        torch.cuda.synchronize()
        results.append((out, h, dy, dg, dr, *dw))
    assert all(torch.equal(a, b) for a, b in zip(*results))
