"""A paged cache, attention over it and the verification of drafted tokens, from their definitions (test infrastructure only): pages as lists that are pushed and popped, attention and sums of
weights in float64, one row at a time."""
from __future__ import annotations

import numpy as np


def extend(page, num_pages, new, kv_len, held, table, stack, num_free, max_rows):
    """State behind the call and the slots of the rows: (kv_len, held, table, num_free, q_start, slots, granted)."""
    n, width = table.shape
    kv_len, held, table = (x.copy() for x in (kv_len, held, table))
    pile = list(stack[:num_free])
    claimed, q_start, granted = 0, [0], []
    slots = np.full(max_rows, -1, dtype=np.int64)
    total = 0
    for i in range(n):
        m = max(int(new[i]), 0)
        start, total = total, total + m
        q_start.append(min(total, max_rows))
        fits = kv_len[i] + m <= width * page and (m == 0 or total <= max_rows)
        need = max(0, -(-int(kv_len[i] + m) // page) - int(held[i])) if fits else 0
        claimed += need
        ok = fits and (need == 0 or claimed <= num_free)
        granted.append(int(ok))
        if not ok:
            continue
        for _ in range(need):
            table[i, held[i]] = pile.pop()
            held[i] += 1
        for j in range(m):
            t = int(kv_len[i]) + j
            number = int(table[i, t // page])
            slots[start + j] = number * page + t % page if 0 <= number < num_pages else -1
        kv_len[i] += m
    return kv_len, held, table, len(pile), np.array(q_start), slots, np.array(granted)


def truncate(page, drop, kv_len, held, table, stack, num_free):
    """(kv_len, held, stack, num_free)."""
    kv_len, held, stack = kv_len.copy(), held.copy(), stack.copy()
    for i in range(len(drop)):
        kv_len[i] = max(0, int(kv_len[i]) - max(0, int(drop[i])))
        keep = min(int(held[i]), -(-int(kv_len[i]) // page))
        for b in range(keep, int(held[i])):
            if num_free < len(stack):
                stack[num_free] = table[i, b]
                num_free += 1
        held[i] = keep
    return kv_len, held, stack, num_free


def attention(q, k_cache, v_cache, table, kv_len, q_start, scale):
    """q [rows, heads, dim], caches [pages, kv_heads, page, dim], float64.  Yields (row, o [heads, dim], lse [heads], weights' sum of |v| [heads, dim], largest scale * sum |q||k| [heads], keys seen)
    for each row of each sequence."""
    heads, kv_heads = q.shape[1], k_cache.shape[1]
    page, G = k_cache.shape[2], heads // kv_heads
    for i, L in enumerate(kv_len):
        n = q_start[i + 1] - q_start[i]
        for j in range(n):
            row, seen = q_start[i] + j, max(0, L - n + j + 1)
            keys = [(table[i, t // page], t % page) for t in range(seen)]
            keys = [(p, r) for p, r in keys if 0 <= p < k_cache.shape[0]]
            o, a = np.zeros(q.shape[1:]), np.zeros(q.shape[1:])
            lse, size = np.full(heads, -np.inf), np.zeros(heads)
            if keys:
                at, of = np.array(keys).T
                for h in range(heads):
                    k, v = k_cache[at, h // G, of], v_cache[at, h // G, of]
                    x = k @ q[row, h] * scale
                    top = x.max()
                    w = np.exp(x - top)
                    lse[h] = top + np.log(w.sum())
                    w /= w.sum()
                    o[h], a[h], size[h] = w @ v, w @ np.abs(v), (np.abs(k) @ np.abs(q[row, h])).max() * scale
            yield row, o, lse, a, size, len(keys)


def verify(target, draft, tokens, count, uniforms, last_uniform):
    """One request: target [drafts + 1, vocab], draft [drafts, vocab] or None, float64.  (accepted, out [drafts + 1])."""
    places, vocab = target.shape
    kept = 0
    while kept < count:
        d = int(tokens[kept])
        if not 0 <= d < vocab:
            break
        p, q = float(target[kept, d]), 1.0 if draft is None else float(draft[kept, d])
        if not (np.isfinite(p) and np.isfinite(q) and float(uniforms[kept]) * q < p):  # (exact: both have 24 bits)
            break
        kept += 1
    p = np.where(np.isfinite(target[kept]) & (target[kept] > 0), target[kept], 0.0)
    w = p
    if kept < count:
        if draft is None:
            w = p.copy()
            if 0 <= tokens[kept] < vocab:
                w[tokens[kept]] = 0.0
        else:
            with np.errstate(invalid="ignore"):
                w = target[kept] - draft[kept]
            w = np.where(np.isfinite(w) & np.isfinite(draft[kept]) & (w > 0), w, 0.0)
        if not w.any():
            w = p
    token = -1
    if w.any():
        running = np.cumsum(w)
        past = np.flatnonzero((running > float(last_uniform) * running[-1]) & (w > 0))
        token = int(past[0]) if len(past) else int(np.flatnonzero(w)[-1])
    return kept, [int(t) for t in tokens[:kept]] + [token] + [-1] * (places - 1 - kept)
