"""Linear attention with a decay for each head in float64, token by token as it is defined (test infrastructure only; torch tensors, any device)."""
from __future__ import annotations

import torch


def _heads(x, n):
    """[tokens, heads, d] -> float64 with every key/value head repeated for its query heads."""
    return x.double().repeat_interleave(n // x.shape[1], 1)


def forward(q, k, v, log_decay, scale, state=None):
    """One sequence: o [tokens, H, d], the state behind it [Hk, d, d], and the sum of its terms' magnitudes."""
    Hk, G = k.shape[1], q.shape[1] // k.shape[1]
    decay = torch.exp(log_decay.double()).view(Hk, 1, 1)
    S = torch.zeros(Hk, k.shape[2], v.shape[2], dtype=torch.float64, device=q.device) if state is None else state.double().clone()
    size, out = S.abs(), []
    for t in range(q.shape[0]):
        add = k[t].double()[:, :, None] * v[t].double()[:, None, :]
        S, size = decay * S + add, decay * size + add.abs()
        out.append(scale * torch.matmul(q[t].double().view(Hk, G, -1), S).flatten(0, 1))
    return torch.stack(out), S, size


def backward(q, k, v, log_decay, scale, d_o, state=None, d_final=None):
    """dq, dk, dv, the gradient of the state before the sequence and the sum of its terms' magnitudes."""
    n, H, Hk = q.shape[0], q.shape[1], k.shape[1]
    G = H // Hk
    decay = torch.exp(log_decay.double()).view(Hk, 1, 1)
    S = torch.zeros(Hk, k.shape[2], v.shape[2], dtype=torch.float64, device=q.device) if state is None else state.double().clone()
    dq = []
    for t in range(n):
        S = decay * S + k[t].double()[:, :, None] * v[t].double()[:, None, :]
        dq.append(scale * torch.matmul(d_o[t].double().view(Hk, G, -1), S.transpose(1, 2)).flatten(0, 1))
    dS = torch.zeros_like(S) if d_final is None else d_final.double().clone()
    size, dk, dv = dS.abs(), [], []
    for t in reversed(range(n)):
        add = scale * torch.matmul(q[t].double().view(Hk, G, -1).transpose(1, 2), d_o[t].double().view(Hk, G, -1))
        dS, size = dS + add, size + scale * torch.matmul(q[t].double().abs().view(Hk, G, -1).transpose(1, 2), d_o[t].double().abs().view(Hk, G, -1))
        dk.append(torch.matmul(dS, v[t].double()[:, :, None])[..., 0])
        dv.append(torch.matmul(k[t].double()[:, None, :], dS)[:, 0])
        dS, size = decay * dS, decay * size
    return torch.stack(dq), torch.stack(dk[::-1]), torch.stack(dv[::-1]), dS, size


def rounding(q, k, v, log_decay, scale, state=None, backwards=False, block=64):
    """Root of the sum of squares of what the kernels hand on in bf16 terms on the way to an output [tokens, heads of q, d]: the weighted scores inside a block of
    rows times v, and the state before the block times q.  q has either all query heads (k, v shared by them) or only the key/value heads (k, v of all
    query heads added up)."""
    n, H = q.shape[0], max(q.shape[1], k.shape[1])
    Hk = min(q.shape[1], k.shape[1])
    out_heads, G = q.shape[1], H // Hk
    lg = log_decay.double().clamp(min=-1e4).repeat_interleave(G).view(H, 1, 1)
    qh, kh, vh = (_heads(x, H).transpose(0, 1) for x in (q, k, v))
    S = torch.zeros(H, k.shape[2], v.shape[2], dtype=torch.float64, device=q.device)
    if state is not None:  # (a query head carries its share)
        S += state.double().repeat_interleave(G, 0) / (G if q.shape[1] == Hk else 1)
    out = torch.zeros(out_heads, n, v.shape[2], dtype=torch.float64, device=q.device)
    starts = list(range(0, n, block))
    for b in reversed(starts) if backwards else starts:
        e = min(n, b + block)
        i = torch.arange(e - b, device=q.device, dtype=torch.float64)
        far = (i[None] - i[:, None]) if backwards else (i[:, None] - i[None])
        P = torch.matmul(qh[:, b:e], kh[:, b:e].transpose(1, 2)) * torch.exp(lg * far.clamp(min=0)) * (far >= 0)
        inner = torch.matmul(P ** 2, vh[:, b:e] ** 2)
        whole = S if out_heads == H else S.view(Hk, G, *S.shape[1:]).sum(1)
        lead = torch.exp(2 * lg[::1 if out_heads == H else G] * ((e - b - 1 - i) if backwards else (i + 1)).view(1, -1, 1))
        outer = lead * torch.matmul((qh if out_heads == H else qh[::G])[:, b:e] ** 2, whole ** 2)
        out[:, b:e] = (inner if out_heads == H else inner.view(Hk, G, *inner.shape[1:]).sum(1)) + outer
        left = torch.exp(lg * ((i + 1) if backwards else (e - b - 1 - i)).view(1, -1, 1))
        S = torch.exp(lg * (e - b)) * S + torch.matmul((kh[:, b:e] * left).transpose(1, 2), vh[:, b:e])
    return scale * out.sqrt().transpose(0, 1)
