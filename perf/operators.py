"""What the operators around chunk attention are timed on: rotary positions of a chunk, the norms around a block with gate and residual
scale, and linear attention with a decay for each head.

A case is a dict of plain values.  `op` says which call one pass makes:

  rope_fwd, rope_bwd   queries and keys of a chunk between the projection's rows and the attention's buffers
  norm_fwd, norm_bwd   residual' = alpha residual + beta act(gate) N(y; post), h = N(residual'; pre)
  lin_fwd, lin_bwd     linear attention over a chunk's sequences, with states where a sequence goes on or comes back
  lin_step             one token for each of a batch of sequences whose states lie in a pool

Chunks follow from `tail` and `context` (a slice of `tail` tokens behind `context` others; 0: none) and from `tokens`, `median`,
`sigma`, `low`, `high` (whole sequences packed behind it, lengths log-normal and clipped, drawn from `lengths_seed`); `lengths` names a
fixed list instead, `batch` stands for so many sequences of one new token each behind contexts of 1 to `context` tokens.
"""
import itertools
import math
import random

import torch

own = False

DEVICE = "cuda"
FIXED_LENGTHS = {"four_short": (256, 512, 128, 128)}
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


# ---- cases ----
def _chunk(tail=0, context=0, tokens=0, median=1024, sigma=1.0, low=128, high=4096, lengths_seed=0, lengths="", batch=0):
    return {"tail": tail, "context": context, "tokens": tokens, "median": median, "sigma": sigma, "low": low, "high": high,
            "lengths_seed": lengths_seed, "lengths": lengths, "batch": batch}


def _rope(name, op, heads, kv_heads, dim, rotary, interleaved=False, base=10000.0, scaling="none", factor=1.0, original=0,
          magnitude=1.0, dk="bf16", **chunk):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "rotary": rotary, "interleaved": interleaved,
            "base": base, "scaling": scaling, "factor": factor, "original": original, "magnitude": magnitude, "dk": dk, **_chunk(**chunk)}


def _norm(name, op, rows, cols, residual="bf16", y=True, gate="none", post=True, pre=True, weights="f32", alpha=1.0, beta=1.0, pad=0):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "residual": residual, "y": y, "gate": gate, "post": post, "pre": pre,
            "weights": weights, "alpha": alpha, "beta": beta, "pad": pad}


def _linear(name, op, heads, kv_heads, dim, **chunk):
    return {"name": name, "op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, **_chunk(**chunk)}


def listed():
    return [
        # one new token for each of 64 sequences: a serving step, bound by the launch
        _rope("rope_64_tokens", "rope_fwd", 32, 8, 128, 128, batch=64, context=32768),
        # tail slice of a 64K sequence packed with short ones, positions scaled by a ramp for a longer context
        _rope("rope_hybrid_64k", "rope_fwd", 32, 8, 128, 128, base=500000.0, scaling="ramp", factor=8.0, original=8192, magnitude=1.2,
              tail=8192, context=57344, tokens=8192, lengths_seed=3),
        # gradients of a skewed packed batch, dK collected in float32; half of each head is rotated, in neighbouring pairs
        _rope("rope_packed_64k_bwd", "rope_bwd", 32, 8, 128, 64, interleaved=True, dk="f32", tokens=65536, median=2048, sigma=1.2,
              high=16384, lengths_seed=4),
        # norms around a block for 64 single tokens
        _norm("norm_64_tokens", "norm_fwd", 64, 4096),
        # the same for a micro-batch of 16K tokens, with a gate
        _norm("norm_16k_gated", "norm_fwd", 16384, 4096, gate="sigmoid", beta=0.5),
        # its gradients at the width of 64 heads, residual stream in float32, a last micro-batch of odd size
        _norm("norm_8k_wide_bwd", "norm_bwd", 8191, 8192, residual="f32", alpha=0.75, beta=0.5),
        # norm of each head of a linear attention's output, gated: short rows, many of them
        _norm("norm_heads_bwd", "norm_bwd", 16384 * 32, 128, residual="none", gate="silu", pre=False, weights="bf16"),
        # four short sequences: the smallest chunk, bound by launches and latency
        _linear("linear_packed_1k_d64", "lin_fwd", 8, 8, 64, lengths="four_short"),
        # a slice of a long sequence: state in, state out
        _linear("linear_slice_8k", "lin_fwd", 32, 32, 128, tail=8192, context=24576),
        # skewed packed batch of 64K tokens: the largest call
        _linear("linear_packed_64k", "lin_fwd", 32, 8, 128, tokens=65536, median=2048, sigma=1.2, high=16384, lengths_seed=4),
        # gradients of a tail slice with a state, packed with short sequences
        _linear("linear_hybrid_16k_bwd", "lin_bwd", 32, 8, 128, tail=8192, context=57344, tokens=8192, lengths_seed=3),
        # a serving step of 128 sequences
        _linear("linear_step_128", "lin_step", 32, 32, 128, batch=128),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _draw_chunk(rng, most):
    kind = rng.choice(["packed", "split", "hybrid"])
    median = _log_uniform(rng, 60, 4096)
    c = _chunk(median=median, sigma=rng.choice([0.5, 1.0, 1.2]), low=rng.choice([1, 33, 128]), high=min(8 * median, 16384), lengths_seed=rng.randint(1, 1 << 30))
    if kind != "split":
        c["tokens"] = _log_uniform(rng, 200, most if kind == "packed" else min(most, 16384))
    if kind != "packed":
        c.update(tail=_log_uniform(rng, 1, min(most, 16384)), context=_log_uniform(rng, 1, 65536))
    return c


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["rope_fwd", "rope_bwd", "norm_fwd", "norm_bwd", "lin_fwd", "lin_bwd", "lin_step"])
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (64, 8), (8, 8), (8, 2), (16, 16), (32, 32)])
    dim = rng.choice([128, 128, 64, 96, 256])
    if op.startswith("rope"):
        interleaved = rng.random() < 0.4
        rotary = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        scaling = rng.choice(["none", "linear", "base", "ramp"]) if rotary > 2 else "none"
        chunk = _draw_chunk(rng, 65536 * 5120 // max(5120, (heads + kv_heads) * dim))
        if rng.random() < 0.2:
            chunk = _chunk(batch=_log_uniform(rng, 1, 1024), context=_log_uniform(rng, 1, 131072))
        case = _rope("", op, heads, kv_heads, dim, rotary, interleaved, rng.choice([10000.0, 500000.0]), scaling,
                     1.0 if scaling == "none" else rng.choice([2.0, 4.5, 16.0]), 4096, rng.choice([1.0, 1.25]),
                     rng.choice(["bf16", "f32"]), **chunk)
    elif op.startswith("norm"):
        cols = rng.choice([4096, 8192, 128, 512, _log_uniform(rng, 8, 2048) * 8, _log_uniform(rng, 3, 16384), 96, 256])
        rows = min(_log_uniform(rng, 1, 1 << 19), (1 << 26) // cols)
        residual, y = rng.choice([("bf16", True), ("f32", True), ("none", True), ("bf16", False), ("f32", False)])
        pre = (residual != "none" and rng.random() < 0.8) or not y
        case = _norm("", op, rows, cols, residual, y, rng.choice(["none", "none", "plain", "sigmoid", "silu"]) if y else "none",
                     y and rng.random() < 0.7, pre, rng.choice(["f32", "bf16"]), rng.choice([1.0, 0.75]),
                     rng.choice([1.0, 0.5]), rng.choice([0, 0, 8, 3]))
    elif op == "lin_step":
        case = _linear("", op, heads, kv_heads, dim, batch=_log_uniform(rng, 1, max(1, (1 << 26) // (kv_heads * dim * dim))))
    else:
        chunk = _draw_chunk(rng, (65536 if op == "lin_fwd" else 16384) * 5120 // max(5120, (heads + kv_heads) * dim) * 128 // max(128, dim))
        case = _linear("", op, heads, kv_heads, dim, **chunk)
    del case["name"]
    return case


# ---- what a chunk is made of ----
def _segments(case):
    """[(q_start, q_len, kv_start, kv_len)] of the chunk."""
    if case["batch"]:
        rng = random.Random(case["batch"] + case["context"])
        lens = [1] * case["batch"]
        longest = min(case["context"], (1 << 27) // (case["kv_heads"] * case["dim"] * case["batch"]))  # (the buffer of keys is kept to a size)
        ctx = [rng.randint(0, longest) for _ in lens]
    else:
        lens = [case["tail"]] * (case["tail"] > 0) + list(FIXED_LENGTHS.get(case["lengths"], ())) + _lengths(case)
        ctx = [case["context"] if case["tail"] and n == 0 else 0 for n in range(len(lens))]
    q = [0, *itertools.accumulate(lens)]
    kv = [0, *itertools.accumulate(c + n for c, n in zip(ctx, lens))]
    return [(q[i], lens[i], kv[i], ctx[i] + lens[i]) for i in range(len(lens))]


def _lengths(case):
    rng = random.Random(case["lengths_seed"])
    drawn = (min(max(int(rng.lognormvariate(math.log(case["median"]), case["sigma"])), case["low"]), case["high"]) for _ in range(case["tokens"] + 1))
    ends = [0, *itertools.takewhile(lambda e: e < case["tokens"], itertools.accumulate(drawn))]
    return [b - a for a, b in zip(ends, [*ends[1:], case["tokens"]]) if b > a]


def _frequencies(case):
    """Angle per position of each pair (float64)."""
    R, s = case["rotary"], case["factor"]
    j = torch.arange(R // 2, dtype=F64, device=DEVICE)
    base = case["base"] * (s ** (R / (R - 2)) if case["scaling"] == "base" else 1.0)
    f = base ** (-2.0 * j / R)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "ramp":
        gamma = ((case["original"] * f / (2.0 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = gamma * f + (1.0 - gamma) * f / s
    return f


# ---- inputs ----
def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    op = case["op"]

    def normal(*shape, dtype=BF16, scale=1.0):
        return torch.randn(shape, generator=gen, device=DEVICE, dtype=F32).mul_(scale).to(dtype)

    state = {"case": case}
    if op.startswith("norm"):
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        rtype = F32 if case["residual"] == "f32" else BF16
        wtype = F32 if case["weights"] == "f32" else BF16

        def padded(dtype=BF16, scale=1.0):
            return normal(rows, cols + pad, dtype=dtype, scale=scale)[:, :cols]

        def like(dtype=BF16):
            return torch.empty((rows, cols), dtype=dtype, device=DEVICE)

        has_r = case["residual"] != "none"
        state.update(y=padded(scale=0.5) if case["y"] else None, gate=padded() if case["gate"] != "none" else None,
                     post=(1.0 + 0.1 * normal(cols, dtype=F32)).to(wtype) if case["post"] else None,
                     pre=(1.0 + 0.1 * normal(cols, dtype=F32)).to(wtype) if case["pre"] else None)
        if op == "norm_fwd":
            state.update(residual=padded(rtype, 2.0) if has_r else None, out=like(rtype) if case["y"] else None, h=like() if case["pre"] else None)
        else:
            state.update(stored=padded(rtype, 2.0) if has_r else None, d_out=padded(rtype) if has_r or not case["pre"] else None,
                         d_h=padded() if case["pre"] else None, dy=like() if case["y"] else None,
                         d_gate=like() if case["gate"] != "none" else None, d_residual=like(rtype) if has_r else None,
                         d_post=torch.empty(cols, device=DEVICE) if case["post"] else None,
                         d_pre=torch.empty(cols, device=DEVICE) if case["pre"] else None)
            if own:
                from paper_2509_21275_amd import fused_norm
                state["ws"] = fused_norm.alloc_workspace(rows, cols, DEVICE)
        return state

    H, Hk, d = case["heads"], case["kv_heads"], case["dim"]
    if op == "lin_step":
        B = case["batch"]
        slots = torch.randperm(B + 1, generator=gen, device=DEVICE)[:B].to(torch.int32)
        log_decay = -torch.exp2(-torch.linspace(4.0, 10.0, Hk, device=DEVICE))
        return {**state, "q": normal(B, H, d), "k": normal(B, Hk, d), "v": normal(B, Hk, d), "o": torch.empty((B, H, d), dtype=BF16, device=DEVICE),
                "log_decay": log_decay, "slots": slots, "states": normal(B + 1, Hk, d, d, dtype=F32, scale=4.0),
                "states_out": torch.zeros((B + 1, Hk, d, d), device=DEVICE), "scale": d ** -0.5}

    segs = _segments(case)
    total, total_kv = segs[-1][0] + segs[-1][1], segs[-1][2] + segs[-1][3]
    lens = torch.tensor([s[1] for s in segs], device=DEVICE)
    seg_of = torch.repeat_interleave(torch.arange(len(segs), device=DEVICE), lens)
    starts, ctx = torch.tensor([s[0] for s in segs], device=DEVICE), torch.tensor([s[3] - s[1] for s in segs], device=DEVICE)
    at = torch.arange(total, device=DEVICE) - starts[seg_of]
    if op.startswith("rope"):
        state.update(freq=_frequencies(case), positions=at + ctx[seg_of], key_rows=at + (ctx + torch.tensor([s[2] for s in segs], device=DEVICE))[seg_of])
        if op == "rope_fwd":  # q, k: rows of one projection that holds queries, keys and values
            qkv = normal(total, H + 2 * Hk, d)
            state.update(q=qkv[:, :H], k=qkv[:, H:H + Hk], q_out=torch.empty((total, H, d), dtype=BF16, device=DEVICE),
                         k_out=torch.zeros((total_kv, Hk, d), dtype=BF16, device=DEVICE))
        else:
            grad = torch.zeros((total, H + 2 * Hk, d), dtype=BF16, device=DEVICE)
            state.update(dq=normal(total, H, d), dk=normal(total_kv, Hk, d, dtype=F32 if case["dk"] == "f32" else BF16),
                         dq_out=grad[:, :H], dk_out=grad[:, H:H + Hk])
        if own:
            import paper_2509_21275_amd as ca
            from paper_2509_21275_amd import chunk_rope
            state["desc"] = ca.make_desc(segs, H, Hk, d, total, total_kv, d ** -0.5)
            state["spec"] = chunk_rope.make_rope(case["rotary"], case["base"], interleaved=case["interleaved"], scaling=case["scaling"],
                                                 factor=case["factor"], original_length=case["original"], low_rotations=1.0,
                                                 high_rotations=32.0, magnitude=case["magnitude"])
        return state

    # linear attention: a slice with context starts from the state of the tokens before it and leaves its own; whole sequences start from nothing
    first = 0 if case["tail"] and case["context"] else -1
    log_decay = -torch.exp2(-torch.linspace(4.0, 10.0, Hk, device=DEVICE))
    state.update(q=normal(total, H, d), k=normal(total, Hk, d), v=normal(total, Hk, d), log_decay=log_decay, scale=d ** -0.5)
    if first == 0:
        state["states"] = normal(1, Hk, d, d, dtype=F32, scale=4.0)
    if op == "lin_fwd":
        state["o"] = torch.empty((total, H, d), dtype=BF16, device=DEVICE)
        if first == 0:
            state["states_out"] = torch.empty((1, Hk, d, d), device=DEVICE)
    else:
        state.update(do=normal(total, H, d), dq=torch.empty((total, H, d), dtype=BF16, device=DEVICE),
                     dk=torch.empty((total, Hk, d), dtype=BF16, device=DEVICE), dv=torch.empty((total, Hk, d), dtype=BF16, device=DEVICE))
        if first == 0:
            state.update(d_states_out=normal(1, Hk, d, d, dtype=F32), d_states=torch.empty((1, Hk, d, d), device=DEVICE))
    # blocks of BLOCK tokens that no sequence border cuts: token of each place, length and sequence of each block, its first token's place in the sequence
    n_blocks = (lens + BLOCK - 1) // BLOCK
    block_seg = torch.repeat_interleave(torch.arange(len(segs), device=DEVICE), n_blocks)
    begin = (torch.arange(len(block_seg), device=DEVICE) - (torch.cumsum(n_blocks, 0) - n_blocks)[block_seg]) * BLOCK
    state["blocks"] = {"seg": block_seg, "begin": begin, "len": (lens[block_seg] - begin).clamp(max=BLOCK), "whole": lens[block_seg],
                       "token": starts[block_seg][:, None] + begin[:, None] + torch.arange(BLOCK, device=DEVICE)[None], "total": total}
    if own:
        from paper_2509_21275_amd import chunk_linear
        state["desc"] = chunk_linear.make_desc([(s[0], s[1], first if n == 0 else -1, first if n == 0 else -1) for n, s in enumerate(segs)],
                                               H, Hk, d, total, 1, d ** -0.5)
        state["ws"] = chunk_linear.alloc_workspace(state["desc"], DEVICE)
    return state


# ---- the passes ----
def run(state):
    case, op = state["case"], state["case"]["op"]
    if op.startswith("rope"):
        return _run_rope(state, case, op)
    if op.startswith("norm"):
        return _run_norm(state, case, op)
    return _run_linear(state, case, op)


def _rotate(x, cos, sin, case, sign):
    """x [rows, heads, dim] in 32 bits, its first `rotary` elements of each head rotated and scaled."""
    R, half = case["rotary"], case["rotary"] // 2
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if case["interleaved"] else (x[..., :half], x[..., half:R])
    u, w = a * cos - sign * b * sin, b * cos + sign * a * sin
    turned = torch.stack((u, w), -1).flatten(-2) if case["interleaved"] else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _run_rope(s, case, op):
    if own:
        from paper_2509_21275_amd import chunk_rope
        if op == "rope_fwd":
            chunk_rope.chunk_rope_fwd(s["desc"], s["spec"], s["q"], s["k"], s["q_out"], s["k_out"])
            return {"q": s["q_out"], "k": s["k_out"]}
        chunk_rope.chunk_rope_bwd(s["desc"], s["spec"], s["dq"], s["dk"], s["dq_out"], s["dk_out"])
        return {"dq": s["dq_out"], "dk": s["dk_out"]}
    angle = s["positions"][:, None].to(F64) * s["freq"][None]
    cos, sin = (f(angle).mul(case["magnitude"]).to(F32)[:, None] for f in (torch.cos, torch.sin))
    if op == "rope_fwd":
        s["q_out"].copy_(_rotate(s["q"].to(F32), cos, sin, case, 1.0))
        s["k_out"][s["key_rows"]] = _rotate(s["k"].to(F32), cos, sin, case, 1.0).to(BF16)
        return {"q": s["q_out"], "k": s["k_out"]}
    s["dq_out"].copy_(_rotate(s["dq"].to(F32), cos, sin, case, -1.0))
    s["dk_out"].copy_(_rotate(s["dk"][s["key_rows"]].to(F32), cos, sin, case, -1.0))
    return {"dq": s["dq_out"], "dk": s["dk_out"]}


EPS = 1e-5


def _gate(g, kind):
    """act(g) and its derivative."""
    if kind == "plain":
        return g, torch.ones_like(g)
    p = torch.sigmoid(g)
    return (p, p * (1.0 - p)) if kind == "sigmoid" else (g * p, p * (1.0 + g * (1.0 - p)))


def _run_norm(s, case, op):
    kind, alpha, beta = case["gate"], case["alpha"], case["beta"]
    if own:
        from paper_2509_21275_amd import fused_norm
        if op == "norm_fwd":
            fused_norm.fused_norm_fwd(s["y"], s["gate"], s["residual"], s["post"], s["pre"], s["out"], s["h"], eps=EPS, gate_kind=kind,
                                      residual_scale=alpha, block_scale=beta)
            return {n: s[n] for n in ("out", "h") if s[n] is not None}
        fused_norm.fused_norm_bwd(s["y"], s["gate"], s["stored"], s["post"], s["pre"], s["d_out"], s["d_h"], s["dy"], s["d_gate"],
                                  s["d_residual"], s["d_post"], s["d_pre"], s["ws"], eps=EPS, gate_kind=kind, residual_scale=alpha,
                                  block_scale=beta)
        return {n: s[n] for n in ("dy", "d_gate", "d_residual", "d_post", "d_pre") if s[n] is not None}
    out = {}
    if s["y"] is not None:
        y = s["y"].to(F32)
        inv_y = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
        w_post = s["post"].to(F32) if case["post"] else None
        normed = y * inv_y * w_post if case["post"] else y
        act, slope = _gate(s["gate"].to(F32), kind) if kind != "none" else (None, None)
    if op == "norm_fwd":
        total = alpha * s["residual"].to(F32) if s["residual"] is not None else 0.0
        if s["y"] is not None:
            total = total + beta * (normed if act is None else normed * act)
            s["out"].copy_(total)
            out["out"] = s["out"]
        if case["pre"]:
            s["h"].copy_(total * torch.rsqrt(total.square().mean(-1, keepdim=True) + EPS) * s["pre"].to(F32))
            out["h"] = s["h"]
        return out
    t = s["d_out"].to(F32) if s["d_out"] is not None else 0.0
    if case["pre"]:
        r, dh = s["stored"].to(F32), s["d_h"].to(F32)
        inv = torch.rsqrt(r.square().mean(-1, keepdim=True) + EPS)
        r = r * inv
        out["d_pre"] = s["d_pre"].copy_((dh * r).sum(0))
        dh = dh * s["pre"].to(F32)
        t = t + inv * (dh - r * (dh * r).mean(-1, keepdim=True))
    if s["d_residual"] is not None:
        out["d_residual"] = s["d_residual"].copy_(alpha * t)
    if s["y"] is not None:
        if act is not None:
            out["d_gate"] = s["d_gate"].copy_(beta * t * normed * slope)
        u = beta * t if act is None else beta * t * act
        if case["post"]:
            y = y * inv_y
            out["d_post"] = s["d_post"].copy_((u * y).sum(0))
            u = u * w_post
            u = inv_y * (u - y * (u * y).mean(-1, keepdim=True))
        out["dy"] = s["dy"].copy_(u)
    return {n: out[n] for n in ("dy", "d_gate", "d_residual", "d_post", "d_pre") if n in out}


BLOCK = 128


def _decayed(q, k, v, lg, b, scale, state, backwards=False):
    """Linear attention of [heads, tokens, dim] tensors in blocks: sums over the tokens up to the own one (backwards: from it on), lg [heads] in 64 bits.
    `state` [heads, dim, dim] is what the first sequence's tokens (backwards: its last ones) add to, and what that sequence leaves is returned."""
    h, n = q.shape[0], len(b["seg"])
    i = torch.arange(BLOCK, device=DEVICE)
    live = i[None] < b["len"][:, None]
    token = torch.where(live, b["token"], b["total"])

    def blocks(x):  # a row of zeros stands where a block has no token
        return torch.cat((x, x.new_zeros(h, 1, x.shape[-1])), 1)[:, token]

    def power(e):  # decay to the power of e, for each head
        return torch.exp(lg.view(-1, *[1] * e.dim()) * e[None].to(F64)).to(F32)

    qb, kb, vb = blocks(q), blocks(k), blocks(v)
    apart = (i[None] - i[:, None]) if backwards else (i[:, None] - i[None])
    o = torch.matmul(torch.matmul(qb, kb.transpose(-1, -2)) * (power(apart.clamp(min=0)) * (apart >= 0))[:, None], vb)
    # what a block adds to the state behind it (backwards: before it), and the states that reach it
    left = (i[None] + 1 if backwards else b["len"][:, None] - 1 - i[None]).clamp(min=0)
    added = torch.matmul((kb * power(left)[..., None]).transpose(-1, -2), vb)
    end = b["begin"] + b["len"]
    gap = (b["begin"][None] - end[:, None]) if backwards else (b["begin"][:, None] - end[None])
    near = (gap >= 0) & (b["seg"][:, None] == b["seg"][None])
    reach = power(gap.clamp(min=0)) * near
    states = torch.matmul(reach, added.flatten(-2)).view_as(added)
    one = b["seg"] == 0
    if state is not None:
        away = b["whole"] - end if backwards else b["begin"]
        states = states + (power(away) * one)[..., None, None] * state[:, None]
    o = o + power((b["len"][:, None] - 1 - i[None] if backwards else i[None] + 1).expand(n, -1).clamp(min=0))[..., None] * torch.matmul(qb, states)
    final = None
    if state is not None:
        rest = b["begin"] if backwards else b["whole"] - end
        final = torch.matmul((power(rest) * one)[:, None], added.flatten(-2)).view_as(state) + power(b["whole"][:1])[..., None] * state
    out = o.new_empty(h, b["total"], o.shape[-1])
    out[:, token[live]] = o[:, live] * scale
    return out, final


def _run_linear(s, case, op):
    H, Hk, G = case["heads"], case["kv_heads"], case["heads"] // case["kv_heads"]
    if own:
        from paper_2509_21275_amd import chunk_linear
        if op == "lin_step":
            chunk_linear.chunk_linear_step(s["q"], s["k"], s["v"], s["log_decay"], s["states"], s["states_out"], s["slots"], s["o"], s["scale"])
            return {"o": s["o"], "states": s["states_out"]}
        if op == "lin_fwd":
            chunk_linear.chunk_linear_fwd(s["desc"], s["q"], s["k"], s["v"], s["log_decay"], s.get("states"), s["o"], s.get("states_out"), s["ws"])
            return {n: s[n] for n in ("o", "states_out") if n in s}
        chunk_linear.chunk_linear_bwd(s["desc"], s["q"], s["k"], s["v"], s["log_decay"], s.get("states"), s["do"], s.get("d_states_out"),
                                      s["dq"], s["dk"], s["dv"], s.get("d_states"), s["ws"])
        return {n: s[n] for n in ("dq", "dk", "dv", "d_states") if n in s}
    lg = s["log_decay"].to(F64)
    if op == "lin_step":
        B, d, slots = case["batch"], case["dim"], s["slots"].long()
        decay = torch.exp(lg).to(F32).view(1, Hk, 1, 1)
        new = s["states"][slots] * decay + s["k"].to(F32)[..., None] * s["v"].to(F32)[..., None, :]
        s["states_out"][slots] = new
        s["o"].copy_(torch.matmul(s["q"].to(F32).view(B, Hk, G, d), new).view(B, H, d) * s["scale"])
        return {"o": s["o"], "states": s["states_out"]}

    def heads(x):  # [tokens, heads, dim] -> [query heads, tokens, dim] in 32 bits
        return x.to(F32).transpose(0, 1).repeat_interleave(H // x.shape[1], 0)

    lgh, b, scale = lg.repeat_interleave(G), s["blocks"], s["scale"]
    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    S = s["states"][0].repeat_interleave(G, 0) if "states" in s else None
    if op == "lin_fwd":
        o, final = _decayed(q, k, v, lgh, b, scale, S)
        s["o"].copy_(o.transpose(0, 1))
        if final is not None:
            s["states_out"][0] = final[::G]
        return {n: s[n] for n in ("o", "states_out") if n in s}
    do = heads(s["do"])
    dq, _ = _decayed(do, v, k, lgh, b, scale, None if S is None else S.transpose(-1, -2))
    # the states that travel backwards hold scale q^T do; a query head carries its share of the key head's
    R = s["d_states_out"][0].repeat_interleave(G, 0) / (scale * G) if S is not None else None
    dv, d_first = _decayed(k, q, do, lgh, b, scale, R, backwards=True)
    dk, _ = _decayed(v, do, q, lgh, b, scale, None if R is None else R.transpose(-1, -2), backwards=True)
    s["dq"].copy_(dq.transpose(0, 1))
    s["dk"].copy_(dk.view(Hk, G, *dk.shape[1:]).sum(1).transpose(0, 1))
    s["dv"].copy_(dv.view(Hk, G, *dv.shape[1:]).sum(1).transpose(0, 1))
    if d_first is not None:
        s["d_states"][0] = d_first.view(Hk, G, *d_first.shape[1:]).sum(1) * scale
    return {n: s[n] for n in ("dq", "dk", "dv", "d_states") if n in s}


# ---- what a pass cannot do without ----
def work(case):
    op = case["op"]
    if op.startswith("norm"):
        n, r = case["rows"] * case["cols"], {"bf16": 2, "f32": 4, "none": 0}[case["residual"]]
        y, g, h = 2 * case["y"], 2 * (case["gate"] != "none"), 2 * case["pre"]
        if op == "norm_fwd":
            out = (r or 2) if case["y"] else 0
            return {"bytes": n * (y + g + r + h + out), "flops": 12 * n}
        d_out = r or (0 if case["pre"] else 2)
        return {"bytes": n * (2 * y + 2 * g + 2 * r + d_out + h), "flops": 24 * n}
    H, Hk, d = case["heads"], case["kv_heads"], case["dim"]
    if op == "lin_step":
        B = case["batch"]
        return {"bytes": B * (4 * H * d + 4 * Hk * d + 8 * Hk * d * d), "flops": B * d * d * (3 * Hk + 2 * H)}
    total = sum(x[1] for x in _segments(case))
    if op.startswith("rope"):
        k = 6 if op == "rope_bwd" and case["dk"] == "f32" else 4
        return {"bytes": total * d * (4 * H + k * Hk), "flops": 3 * total * d * (H + Hk)}
    states = 2 * 4 * Hk * d * d * bool(case["tail"] and case["context"])
    if op == "lin_fwd":
        return {"bytes": total * d * (4 * H + 4 * Hk) + states, "flops": total * d * d * (2 * H + 2 * Hk)}
    return {"bytes": total * d * (6 * H + 8 * Hk) + 2 * states, "flops": total * d * d * (6 * H + 4 * Hk)}


# ---- the definitions in 64 bits ----
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op.startswith("rope"):
        return _exact_rope(s, case, op)
    if op.startswith("norm"):
        return _exact_norm(s, case, op)
    return _exact_linear(s, case, op)


def _exact_rope(s, case, op):
    R, inter = case["rotary"], case["interleaved"]
    first = torch.arange(0, R, 2, device=DEVICE) if inter else torch.arange(R // 2, device=DEVICE)
    second = first + (1 if inter else R // 2)
    turn = torch.polar(torch.full((), case["magnitude"], dtype=F64, device=DEVICE), s["freq"] * s["positions"][:, None].to(F64))[:, None]
    turn = turn if op == "rope_fwd" else turn.conj()

    def turned(x, into):
        x = x.to(F64)
        z = torch.complex(x[..., first], x[..., second]) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return into.copy_(x) if into is not None else x

    if op == "rope_fwd":
        k = s["k_out"].to(F64)
        k[s["key_rows"]] = turned(s["k"], None)
        return {"q": turned(s["q"], None), "k": k}
    return {"dq": turned(s["dq"], None), "dk": turned(s["dk"][s["key_rows"]], None)}


def _exact_norm(s, case, op):
    def wide(n):
        return s[n].to(F64).requires_grad_(op == "norm_bwd") if s.get(n) is not None else None

    def rms(x, w):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w

    y, gate, post, pre = (wide(n) for n in ("y", "gate", "post", "pre"))
    block = None
    if y is not None:
        block = case["beta"] * (rms(y, post) if post is not None else y)
        if gate is not None:
            block = block * {"plain": lambda g: g, "sigmoid": torch.sigmoid, "silu": lambda g: g / (1.0 + torch.exp(-g))}[case["gate"]](gate)
    if op == "norm_fwd":
        r = wide("residual")
        total = (0.0 if r is None else case["alpha"] * r) + (0.0 if block is None else block)
        return {**({"out": total} if s["out"] is not None else {}), **({"h": rms(total, pre)} if pre is not None else {})}
    # the gradient that arrives at the stored sum, and from there at its two terms
    names, out = [("d_pre", pre)], {}
    t = s["d_out"].to(F64) if s["d_out"] is not None else 0.0
    if pre is not None:
        stored = wide("stored")
        more, out["d_pre"] = torch.autograd.grad(rms(stored, pre), (stored, pre), s["d_h"].to(F64))
        t = t + more
    if s["d_residual"] is not None:
        out["d_residual"] = case["alpha"] * t
    if block is not None:
        names = [(n, x) for n, x in (("dy", y), ("d_gate", gate), ("d_post", post)) if x is not None]
        out.update(zip([n for n, _ in names], torch.autograd.grad(block, [x for _, x in names], t)))
    return {n: out[n] for n in ("dy", "d_gate", "d_residual", "d_post", "d_pre") if n in out}


def _exact_linear(s, case, op):
    H, Hk, G, d, scale = case["heads"], case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], s["scale"]
    lg = s["log_decay"].to(F64).tolist()
    if op == "lin_step":
        states, o = s["states_out"].to(F64), torch.empty(s["o"].shape, dtype=F64, device=DEVICE)
        for b, slot in enumerate(s["slots"].tolist()):
            for h in range(Hk):
                new = math.exp(lg[h]) * s["states"][slot, h].to(F64) + torch.outer(s["k"][b, h].to(F64), s["v"][b, h].to(F64))
                states[slot, h] = new
                o[b, h * G:(h + 1) * G] = scale * s["q"][b, h * G:(h + 1) * G].to(F64) @ new
        return {"o": o, "states": states}
    back = op == "lin_bwd"
    out = {n: torch.empty(s[n].shape, dtype=F64, device=DEVICE) for n in ("o", "states_out", "dq", "dk", "dv", "d_states") if n in s}
    for n, (at, length, _, _) in enumerate(_segments(case)):
        rows = slice(at, at + length)
        i = torch.arange(length, device=DEVICE, dtype=F64)
        for h in range(Hk):
            k, v = (s[x][rows, h].to(F64).requires_grad_(back) for x in ("k", "v"))
            S = s["states"][0, h].to(F64).requires_grad_(back) if n == 0 and "states" in s else None
            if S is not None:
                final = math.exp(lg[h] * length) * S + (k * torch.exp(lg[h] * (length - 1 - i))[:, None]).T @ v
                if not back:
                    out["states_out"][0, h] = final
                else:
                    grads = torch.autograd.grad(final, (k, v, S), s["d_states_out"][0, h].to(F64))
            sums = [0.0, 0.0, 0.0] if S is None or not back else list(grads)
            for g in range(h * G, (h + 1) * G):
                q = s["q"][rows, g].to(F64).requires_grad_(back)
                step = max(1, (1 << 28) // length)
                for r in range(0, length, step):  # rows in slabs: all pairs of a long sequence at once would not fit
                    some = slice(r, min(length, r + step))
                    weight = torch.exp(lg[h] * (i[some, None] - i[None]).clamp(min=0)).tril_(r) * scale
                    o = ((q[some] @ k.T) * weight) @ v
                    if S is not None:
                        o = o + scale * torch.exp(lg[h] * (i[some] + 1))[:, None] * (q[some] @ S)
                    if not back:
                        out["o"][rows, g][some] = o
                        continue
                    given = (q, k, v) if S is None else (q, k, v, S)
                    parts = torch.autograd.grad(o, given, s["do"][rows, g][some].to(F64))
                    out["dq"][rows, g][some] = parts[0][some]
                    sums = [a + b for a, b in zip(sums, parts[1:] if S is not None else (*parts[1:], 0.0))]
            if back:
                out["dk"][rows, h], out["dv"][rows, h] = sums[0], sums[1]
                if S is not None:
                    out["d_states"][0, h] = sums[2]
    return out
