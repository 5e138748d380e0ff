"""Attention of new tokens over a paged cache and a step's bookkeeping, in 64 bits and whole numbers, with
bounds of what the kernels may be off by."""
import math

import torch

BF16, FP32 = 2.0 ** -8, 2.0 ** -24  # half a step


def attention(q, k, v, causal, scale):
    """q [n, G, D], k and v [keys, D], 64 bits: (o, bound of o, lse, bound of lse), [n, G, ...].

    The kernel's scores are sums of D products in 32 bits and come off by at most e = D 2^-23 sum |q k| scale
    (and their place beside the maximum by 2^-23 of either); weights are rounded to bf16 before they meet v, sums over
    keys and the output's division are 32 bits, the output is rounded to bf16.  With A = sum of
    p |v|:  |do| <= 2^-8 (A + |o|) + 2 e A + 2^-18 A;  |dlse| <= e + 2^-20 (1 + |lse|)."""
    n, G, D = q.shape
    if not k.shape[0]:
        zero = torch.zeros((n, G), dtype=torch.float64)
        return torch.zeros_like(q), torch.zeros_like(q), zero - math.inf, zero
    s = torch.einsum("ngd,kd->ngk", q, k) * scale
    size = torch.einsum("ngd,kd->ngk", q.abs(), k.abs()) * scale
    if causal:
        hidden = torch.arange(k.shape[0]) > torch.arange(n)[:, None, None] + (k.shape[0] - n)
        s = s.masked_fill(hidden, -math.inf)
        size = size.masked_fill(hidden, 0)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.clamp(min=-1e300)[..., None])
    o, A = torch.einsum("ngk,kd->ngd", p, v), torch.einsum("ngk,kd->ngd", p, v.abs())
    top = s.masked_fill(torch.isinf(s), 0).abs().amax(-1)
    e = D * 2 * FP32 * size.amax(-1) + 4 * FP32 * top
    bo = 1.01 * BF16 * (A + o.abs()) + (2 * e[..., None] + 2.0 ** -18) * A
    return o, bo, lse, e + 2.0 ** -20 * (1 + lse.masked_fill(torch.isinf(lse), 0).abs())


def gathered(cache, rows, n, layout):
    """[n, Hkv, D] in 64 bits of the first n keys of pages `rows`; a page that there is not reads as zeros."""
    c = cache if layout == "nhd" else cache.transpose(1, 2)
    page = c.shape[1]
    out = torch.zeros((len(rows) * page, *c.shape[2:]), dtype=torch.float64)
    for i, r in enumerate(rows):
        if 0 <= r < c.shape[0]:
            out[i * page:(i + 1) * page] = c[r].double()
    return out[:n]


def chunk(q, k_cache, v_cache, table, cu, lens, causal, scale, layout):
    """(o, bound, lse, bound) of every token: [T, Hq, D] and [Hq, T]; NaN for padding."""
    T, Hq, D = q.shape
    Hkv = k_cache.shape[2 if layout == "nhd" else 1]
    page = k_cache.shape[1 if layout == "nhd" else 2]
    G = Hq // Hkv
    o, bo = (torch.full((T, Hq, D), math.nan, dtype=torch.float64) for _ in range(2))
    lse, bl = (torch.full((Hq, T), math.nan, dtype=torch.float64) for _ in range(2))
    for b in range(len(lens)):
        first, last = cu[b], cu[b + 1]
        n = max(0, min(lens[b], table.shape[1] * page))
        rows = table[b, :-(-n // page)].tolist()
        k, v = gathered(k_cache, rows, n, layout), gathered(v_cache, rows, n, layout)
        for h in range(Hkv if last > first else 0):
            at = slice(h * G, (h + 1) * G)
            r = attention(q[first:last, at].double(), k[:, h], v[:, h], causal, scale)
            o[first:last, at], bo[first:last, at], lse[at, first:last], bl[at, first:last] = r[0], r[1], r[2].T, r[3].T
    return o, bo, lse, bl


def pages(n, page):
    return -(-n // page)


def plan(new, lens, table, free, count, T, page, num_pages):
    """The step's bookkeeping request by request, in lists: cu, seqlens, positions, slots, granted, and the
    updated table, free list and count."""
    table, free = [list(r) for r in table], list(free)
    rows = len(table[0]) * page
    lens = [max(0, min(x, rows)) for x in lens]
    count = max(0, min(count, num_pages))
    stack = free[:count]
    for b, n in enumerate(new):
        if n < 0:
            stack += table[b][:pages(lens[b], page)]
    stack = stack[:num_pages]
    room, asked, total, cu, out, granted, positions, slots = len(stack), 0, 0, [0], [], [], [0] * T, [-1] * T
    for b, n in enumerate(new):
        first = total
        total += max(n, 0)
        cu.append(min(total, T))
        if n < 0:
            out.append(0)
            granted.append(0)
            continue
        need = pages(lens[b] + n, page) - pages(lens[b], page)
        ok = lens[b] + n <= rows and total <= T
        asked += need if ok else 0
        if not ok or (need and asked > room):
            out.append(lens[b])
            granted.append(0)
            continue
        for j in range(need):
            table[b][pages(lens[b], page) + j] = stack.pop()
        out.append(lens[b] + n)
        granted.append(n)
        for i in range(n):
            p = lens[b] + i
            at = table[b][p // page]
            positions[first + i] = p
            slots[first + i] = at * page + p % page if 0 <= at < num_pages else -1
    for i in range(count, len(stack)):
        free[i] = stack[i]
    return cu, out, positions, slots, granted, table, free, len(stack)
