"""Gradients of gates that are wide open or shut, against float64.

Tolerance: relative only.  Half a step of bf16, 2^-8, and for the dozen float32 operations before it, of which exp(-|g|) is off by |g| / ln 2 units of 2^-24 for the rounding of its argument
(g = 80: 116) and the sum over a row of 300 squares by at most 300: 2^-15.  Below 2^-126 the numbers of bf16 are 2^-133 apart (the smallest normal number's
step, 2^-126 * 2^-7), whatever their value, and half a step is 2^-134: at g = 78, exp(-g) = 2^-112.5, a small y times a small gradient gets there."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
@pytest.mark.parametrize("with_norm", [False, True])
def test_gradient_of_an_open_gate(kind, with_norm):
    from paper_2509_21275_amd import fused_norm as fn
    rows, cols, eps = 64, 300, 1e-5
    gen = torch.Generator().manual_seed(5)
    y, t = (torch.randn((rows, cols), generator=gen).to(torch.bfloat16).cuda() for _ in range(2))
    gate = torch.linspace(4.0, 80.0, rows * cols).view(rows, cols)[:, torch.randperm(cols, generator=gen)].to(torch.bfloat16).cuda()
    post = (1 + 0.3 * torch.randn(cols, generator=gen)).cuda() if with_norm else None
    for sign in (1.0, -1.0):
        g = gate * sign
        d_gate = torch.empty_like(y)
        fn.fused_norm_bwd(y, g, None, post, None, t, None, None, d_gate, None, None, None, None, eps=eps, gate_kind=kind)
        torch.cuda.synchronize()
        x, n = g.double(), y.double()
        if with_norm:
            n = n / torch.sqrt((n * n).mean(-1, keepdim=True) + eps) * post.double()
        p, q = 1.0 / (1.0 + torch.exp(-x)), 1.0 / (1.0 + torch.exp(x))  # q = 1 - p, with all its digits
        want = t.double() * n * (p * q if kind == "sigmoid" else p * (1.0 + x * q))
        over = (d_gate.double() - want).abs() - (2.0 ** -8 + 2.0 ** -15) * want.abs() - 2.0 ** -134
        assert float(over.max()) <= 0, (sign, float(x[over > 0].abs().min()), int((over > 0).sum()))
