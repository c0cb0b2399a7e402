"""Plain counterparts of the calls around the cache: places for new tokens one after the other, heads and attention in 64 bits."""
import math

import torch


def place(S, table, lens, new, free, free_count, rows, shared=None, nxt=None, freed=None, freed_count=None, capacity=None):
    """Lists in, a dict of lists out; the stack's entries at and beyond its count are not told."""
    table, lens, B = [list(r) for r in table], list(lens), len(lens)
    width = len(table[0])
    stack = list(free[:free_count])
    capacity = len(free) if capacity is None else capacity
    nxt_of = list(lens if nxt is None else nxt)

    def push(page):
        if len(stack) < capacity:
            stack.append(page)

    for b in range(B):
        for i in range(freed_count[b] if freed is not None else 0):
            push(freed[b][i])
    for b in range(B):
        if new[b] < 0:
            for p in range(-(-lens[b] // S)):
                if p >= (shared[b] if shared else 0):
                    push(table[b][p])
                table[b][p] = -1
            lens[b] = nxt_of[b] = 0
    positions, slots, starts, placed, closed = [], [], [0], [], False
    for b in range(B):
        t = max(new[b], 0)
        starts.append(starts[-1] + t)
        have, pages = -(-lens[b] // S), -(-(lens[b] + t) // S)
        ok = pages <= width and starts[-1] <= rows
        if ok and pages > have:
            closed = closed or len(stack) < pages - have  # from here on nobody gets pages
            ok = not closed
        placed.append(t if ok else 0)
        if not ok:
            positions += [-1] * t
            slots += [-1] * t
            continue
        for p in range(have, pages):
            table[b][p] = stack.pop()
        for i in range(t):
            at = lens[b] + i
            slots.append(table[b][at // S] * S + at % S)
            positions.append(nxt_of[b] + i)
        lens[b] += t
        nxt_of[b] += t
    pad = [-1] * rows
    return dict(table=table, seq_lens=lens, next=nxt_of, placed=placed, token_starts=starts, positions=(positions + pad)[:rows],
                slots=(slots + pad)[:rows], stack=stack)


def heads(x, weight, eps, position, f, magnitude, interleaved):
    """[rows, heads, D] of any type -> float64, and for each element the size that its errors go by."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    R = 2 * f.numel()
    size = y.abs()
    if R:
        a = position.double()[:, None, None] * f.double()
        c, s = magnitude * torch.cos(a), magnitude * torch.sin(a)
        lo, hi = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
        y0, y1 = y[..., lo].clone(), y[..., hi].clone()
        y[..., lo], y[..., hi] = y0 * c - y1 * s, y0 * s + y1 * c
        size[..., lo] = size[..., hi] = (y0.abs() + y1.abs()) * max(magnitude, 1.0)
    return y, size


def attend(q, k_cache, v_cache, table, lens, scale=None):
    """Dense attention of every sequence in float64: out, lse, and for each output the sum of p |v| and for each row the largest sum of |q k| (scaled)."""
    B, H, D = q.shape
    Hkv, S = k_cache.shape[1:3]
    G = H // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    out, terms = torch.zeros(B, H, D, dtype=torch.float64), torch.zeros(B, H, D, dtype=torch.float64)
    lse, reach = torch.full((B, H), -math.inf, dtype=torch.float64), torch.zeros(B, H, dtype=torch.float64)
    for b, n in enumerate(lens):
        n = int(n)
        ids = table[b, :-(-n // S)].long()
        ok = (ids >= 0) & (ids < k_cache.shape[0])
        tok = (ok[:, None] & (torch.arange(ids.numel() * S).view(-1, S) < n)).reshape(-1)
        if not bool(tok.any()):
            continue
        ids = ids.clamp(0, k_cache.shape[0] - 1)
        for h in range(Hkv):
            k, v = (x[ids, h].reshape(-1, D)[tok].double() for x in (k_cache, v_cache))
            x = q[b, h * G:(h + 1) * G].double()
            s = x @ k.T * scale
            reach[b, h * G:(h + 1) * G] = (x.abs() @ k.abs().T * scale).amax(-1)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(s, -1)
            p = torch.softmax(s, -1)
            out[b, h * G:(h + 1) * G] = p @ v
            terms[b, h * G:(h + 1) * G] = p @ v.abs()
    return out, lse, terms, reach
