"""Linear attention at the edges of what a call may be: gradients of states in place where no sequence is cut."""
import pytest
import torch

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
