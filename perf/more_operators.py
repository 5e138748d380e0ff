"""Cases of the operators around a paged cache in serving, and of rotary positions with several axes.

A case is a dict of plain values.  ``kind`` names the operator:

* ``chunk``       attention of each request's new tokens over its keys in a paged cache
* ``plan``        a step's block tables, positions and cache slots from the requests' lengths
* ``axes``        a packed QKV projection to q, k (RMS norm per head, rotation) and v, where each pair of
                  a head turns by the position on one of several axes (time, height, width)
* ``axes_cache``  its serving form: k and v go to their slots of a cache
* ``axes_bwd``    its gradients: the projection's and the two norm weights'

The lengths of a batch are a fixed set for a case, so that its work does not depend on the seed,
which only orders them.
"""
import math
import random

import torch

own = False  # True: run() calls the library; False: elementary torch operations in 32 bits

DEV = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------ the cases
def _chunk(B, q_lo, q_hi, c_lo, c_hi, Hq, Hkv, D, page, layout, causal=True, lse=False, long_q=0, long_c=0):
    """B requests of q_lo to q_hi new tokens after c_lo to c_hi that are in the cache (evenly spaced),
    and with long_q one more of long_q tokens after long_c."""
    return {"kind": "chunk", "B": B, "q_lo": q_lo, "q_hi": q_hi, "c_lo": c_lo, "c_hi": c_hi, "Hq": Hq, "Hkv": Hkv, "D": D,
            "page": page, "layout": layout, "causal": causal, "lse": lse, "long_q": long_q, "long_c": long_c}


def _plan(B, n_lo, n_hi, l_lo, l_hi, page, over=0, pad=0):
    """B requests of n_lo to n_hi new tokens after l_lo to l_hi (spaced over the logarithm); of every
    `over` requests one is over and gives its pages back; pad: tokens of the step's buffers beyond the last."""
    return {"kind": "plan", "B": B, "n_lo": n_lo, "n_hi": n_hi, "l_lo": l_lo, "l_hi": l_hi, "page": page, "over": over, "pad": pad}


def _axes(kind, T, Hq, Hkv, D, R, S, axes, spread, interleaved, weights, P):
    """T tokens; S > 0: T / S sequences of S tokens, q, k, v [B, H, S, D]; S = 0: packed tokens [T, H, D].
    spread: "blocks" (an axis' pairs side by side) or "turns" (pair i has axis i mod axes)."""
    return {"kind": kind, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "R": R, "S": S, "axes": axes, "spread": spread,
            "interleaved": interleaved, "weights": weights, "P": P}


def _axes_cache(T, Hq, Hkv, D, R, page, layout, axes, spread, interleaved, weights, P):
    return dict(_axes("axes_cache", T, Hq, Hkv, D, R, 0, axes, spread, interleaved, weights, P), page=page, layout=layout)


def listed():
    named = [
        # one user's next token after a short prompt: latency
        ("chunk_one_token", _chunk(1, 1, 1, 499, 499, 32, 8, 128, 16, "nhd")),
        # the next tokens of a batch: the cache's bandwidth
        ("chunk_decode_b16", _chunk(16, 1, 1, 4095, 8191, 32, 8, 128, 16, "nhd")),
        # drafted tokens of many requests, checked in one pass; 64-wide heads
        ("chunk_drafts_d64", _chunk(48, 3, 6, 200, 4000, 16, 2, 64, 32, "hnd", lse=True)),
        # a step of a busy server: one prompt's chunk among next tokens, odd sizes
        ("chunk_mixed_step", _chunk(31, 1, 1, 100, 12000, 32, 8, 128, 64, "hnd", long_q=481, long_c=2500)),
        # a long prompt's chunk late in the prompt; the largest case
        ("chunk_2048_after_30000", _chunk(1, 2048, 2048, 30000, 30000, 32, 8, 128, 16, "nhd")),
        # the next tokens of a few requests
        ("plan_4_requests", _plan(4, 1, 1, 10, 3000, 16)),
        # a step of a busy server: next tokens, prompts' chunks, requests that end, a padded buffer
        ("plan_256_requests", _plan(256, 1, 512, 1, 20000, 16, over=17, pad=1000)),
        # many requests with prompts
        ("plan_4096_requests", _plan(4096, 1, 64, 1, 8000, 64, over=50)),
        # image and video tokens of a training batch between projection and attention
        ("axes_b4_s2048", _axes("axes", 8192, 32, 8, 128, 128, 2048, 3, "blocks", False, "bf16", 4096)),
        # the backward pass of the same
        ("axes_bwd_b4_s2048", _axes("axes_bwd", 8192, 32, 8, 128, 128, 2048, 3, "blocks", False, "bf16", 4096)),
        # a packed batch of images, half of each head rotated, axes in turns
        ("axes_bwd_packed_odd", _axes("axes_bwd", 1111, 16, 2, 64, 32, 0, 2, "turns", True, "fp32", 300)),
        # an image in a prompt's chunk, into a paged cache
        ("axes_cache_step", _axes_cache(579, 32, 8, 128, 128, 64, "hnd", 3, "turns", False, "bf16", 32768)),
    ]
    return [dict(c, name=n) for n, c in named]


MOST_SCORES = 1.9e9  # a drawn case's most scores (the largest listed case has 2.03e9)
MOST_KEYS = 9.0e7  # its most values of the keys that it reads (the listed batch has 1.0e8)
MOST_VALUES = 4.0e7  # and the most values of a projection (the listed case has 5.0e7)
MOST_TOKENS = 60000  # and the most tokens of a plan (the listed case has about 63000)


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


HEADS = ((32, 8), (32, 8), (32, 32), (64, 8), (16, 2), (28, 4), (40, 8), (8, 1), (6, 3))


def _draw_once(rng):
    kind = rng.choice(("chunk",) * 6 + ("plan",) * 2 + ("axes", "axes_bwd", "axes_cache"))
    D = rng.choice((64, 128, 128))
    Hq, Hkv = rng.choice(HEADS)
    if kind == "chunk":
        use = rng.choice(("next", "drafts", "prompts", "mixed"))
        page, layout = rng.choice((8, 16, 16, 32, 64, 128, 192, 256)), rng.choice(("nhd", "hnd"))
        c_hi = _log(rng, 1, 32768)
        c_lo = rng.choice((0, c_hi, _log(rng, 1, c_hi)))
        lse, causal = rng.random() < 0.3, rng.random() < 0.9
        if use == "next":
            return _chunk(_log(rng, 1, 128), rng.choice((0, 1, 1)), 1, c_lo, c_hi, Hq, Hkv, D, page, layout, causal, lse)
        if use == "drafts":
            return _chunk(_log(rng, 1, 64), rng.randint(1, 3), rng.randint(3, 9), c_lo, c_hi, Hq, Hkv, D, page, layout, causal, lse)
        if use == "prompts":
            q_hi = _log(rng, 2, 4096)
            return _chunk(_log(rng, 1, 6), rng.choice((q_hi, _log(rng, 1, q_hi))), q_hi, rng.choice((0, c_lo)), c_hi, Hq, Hkv, D,
                          page, layout, causal, lse)
        return _chunk(_log(rng, 1, 64), 1, 1, c_lo, c_hi, Hq, Hkv, D, page, layout, True, lse, _log(rng, 16, 2048),
                      rng.choice((0, _log(rng, 1, 16384))))
    if kind == "plan":
        B, n_hi, l_hi = _log(rng, 1, 4096), _log(rng, 1, 2048), _log(rng, 1, 32768)
        return _plan(B, rng.choice((0, 1, n_hi)), n_hi, rng.choice((0, 1, l_hi)), l_hi, rng.choice((8, 16, 16, 32, 64, 128)),
                     rng.choice((0, 0, 5, 40)), rng.choice((0, _log(rng, 1, 4096))))
    R = rng.choice((D, D, D // 2, 16, 3 * D // 4))
    axes, spread = rng.choice((1, 2, 3, 3, 4)), rng.choice(("blocks", "turns"))
    interleaved, weights, P = rng.random() < 0.4, rng.choice(("bf16", "bf16", "fp32")), _log(rng, 64, 32768)
    if kind == "axes_cache":
        page = rng.choice((8, 16, 16, 32, 64, 192, 4096))
        return _axes_cache(_log(rng, 1, 8192), Hq, Hkv, D, R, page, rng.choice(("nhd", "hnd")), axes, spread, interleaved, weights, P)
    if rng.random() < 0.5:
        S = _log(rng, 1, 8192)
        return _axes(kind, S * _log(rng, 1, 8), Hq, Hkv, D, R, S, axes, spread, interleaved, weights, P)
    return _axes(kind, _log(rng, 1, 32768), Hq, Hkv, D, R, 0, axes, spread, interleaved, weights, P)


def draw(rng: random.Random):
    while True:
        c = _draw_once(rng)
        if c["kind"] == "chunk":
            ql, kl = _lengths(c)
            scores = c["Hq"] * sum(_pairs(a, b, c["causal"]) for a, b in zip(ql, kl))
            size = max(scores / MOST_SCORES, sum(kl) * c["Hkv"] * c["D"] / MOST_KEYS)
            if not sum(ql):
                continue
        elif c["kind"] == "plan":
            n, _ = _plan_lengths(c)
            size = (sum(max(x, 0) for x in n) + c["pad"]) / MOST_TOKENS
            if not sum(max(x, 0) for x in n):
                continue
        else:
            size = c["T"] * c["D"] * (c["Hq"] + 2 * c["Hkv"]) / MOST_VALUES
        if size <= 1:
            return c


# ------------------------------------------------------------------ lengths and work
def _spaced(B, lo, hi):
    return [lo + round((hi - lo) * i / (B - 1)) for i in range(B)] if B > 1 else [hi]


def _lengths(case, seed=0):
    """New tokens and keys (with them) of each request of a chunk: fixed pairs, in an order of the seed's."""
    q, c = _spaced(case["B"], case["q_lo"], case["q_hi"]), _spaced(case["B"], case["c_lo"], case["c_hi"])
    random.Random(1).shuffle(c)
    both = [(a, a + b) for a, b in zip(q, c)]
    if case["long_q"]:
        both.append((case["long_q"], case["long_q"] + case["long_c"]))
    random.Random(seed).shuffle(both)
    return [a for a, _ in both], [b for _, b in both]


def _spaced_log(B, lo, hi):
    return [round(math.exp(math.log(lo + 1) + (math.log(hi + 1) - math.log(lo + 1)) * i / max(B - 1, 1))) - 1 for i in range(B)]


def _plan_lengths(case, seed=0):
    """New tokens (-1: the request is over) and tokens in the cache of each request of a plan."""
    n, old = _spaced_log(case["B"], case["n_lo"], case["n_hi"]), _spaced_log(case["B"], case["l_lo"], case["l_hi"])
    random.Random(1).shuffle(old)
    both = list(zip(n, old))
    if case["over"]:
        both = [(-1, b) if i % case["over"] == case["over"] - 1 else (a, b) for i, (a, b) in enumerate(both)]
    random.Random(seed).shuffle(both)
    return [a for a, _ in both], [b for _, b in both]


def _pairs(sq, skv, causal):
    """Visible (query, key) pairs: query i sees keys up to i + skv - sq."""
    if not causal:
        return sq * skv
    n = min(sq, skv)  # rows that see a key; the last sees skv
    return n * skv - n * (n - 1) // 2


def _pages(n, page):
    return -(-n // page)


def work(case):
    kind = case["kind"]
    if kind == "chunk":
        D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
        ql, kl = _lengths(case)
        rows = sum(ql) * Hq
        keys = sum(k for q, k in zip(ql, kl) if q)
        # read q, and the keys and values of requests with new tokens, with their pages; write o
        b = rows * D * 4 + keys * Hkv * D * 4 + 4 * sum(_pages(k, case["page"]) for k in kl) + 8 * len(ql)
        if case["lse"]:
            b += 4 * rows
        return {"bytes": b, "flops": 4 * D * Hq * sum(_pairs(q, k, case["causal"]) for q, k in zip(ql, kl))}
    if kind == "plan":
        n, old = _plan_lengths(case)
        new = sum(max(x, 0) for x in n)
        page = case["page"]
        taken = sum(_pages(a + b, page) - _pages(b, page) for a, b in zip(n, old) if a > 0)
        given = sum(_pages(b, page) for a, b in zip(n, old) if a < 0)
        # read the lengths, the pages taken, given back and written to; write the lengths, offsets, grants,
        # the tables' new entries, the free list's, positions and slots
        b = 20 * case["B"] + 8 * taken + 8 * given + 4 * sum(a > 0 for a in n) + 8 * (new + case["pad"])
        return {"bytes": b, "flops": 6 * (new + case["pad"]) + 20 * case["B"]}
    D, Hq, Hkv, T, R = case["D"], case["Hq"], case["Hkv"], case["T"], case["R"]
    normed, values = T * (Hq + Hkv) * D, T * (Hq + 2 * Hkv) * D
    wbytes = 2 * D * (2 if case["weights"] == "bf16" else 4)
    # the tables' rows that can occur, and the positions
    b = min(T * case["axes"], case["P"]) * R * 4 + wbytes + 4 * T * case["axes"]
    if kind == "axes":
        return {"bytes": b + 2 * 2 * values, "flops": 9 * normed}
    if kind == "axes_cache":
        return {"bytes": b + 4 * T + 2 * 2 * values, "flops": 9 * normed}
    # read dq, dk, dv and the projection's q and k parts; write its gradient and the weights'
    return {"bytes": b + 2 * (2 * values + normed) + 8 * D, "flops": 16 * normed}


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, std=1.0):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    return t if std == 1.0 else t.mul_(std)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pair_axis(case):
    """The axis of each of a head's rotated pairs."""
    half, axes = case["R"] // 2, case["axes"]
    if case["spread"] == "turns":
        return tuple(i % axes for i in range(half))
    return tuple(min(i * axes // half, axes - 1) for i in range(half))


def _prepare_chunk(case, seed, gen):
    ql, kl = _lengths(case, seed)
    page, D, Hq, Hkv = case["page"], case["D"], case["Hq"], case["Hkv"]
    per = [_pages(k, page) for k in kl]
    pages = sum(per) + 3
    shape = (pages, page, Hkv, D) if case["layout"] == "nhd" else (pages, Hkv, page, D)
    s = {"case": case, "ql": ql, "kl": kl, "k_cache": _normal(gen, shape), "v_cache": _normal(gen, shape)}
    s["q"] = _normal(gen, (sum(ql), Hq, D))
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(kl), max(max(per), 1)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(per):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"] = table
    s["cu_q"] = _ints([sum(ql[:i]) for i in range(len(ql) + 1)])
    s["lens"] = _ints(kl)
    return s


def _prepare_plan(case, seed, gen):
    n, old = _plan_lengths(case, seed)
    page = case["page"]
    held = [_pages(b, page) for b in old]
    taken = sum(_pages(a + b, page) - _pages(b, page) for a, b in zip(n, old) if a > 0)
    pages = sum(held) + taken + 5
    most = max(_pages(max(a, 0) + b, page) for a, b in zip(n, old)) + 1
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    rows = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor(held, device=DEV))
    first = torch.cumsum(torch.tensor([0] + held[:-1], device=DEV), 0)
    table = torch.full((len(n), most), -1, dtype=torch.int32, device=DEV)
    table[rows, torch.arange(len(rows), device=DEV) - first[rows]] = order[:len(rows)]
    free = torch.zeros(pages, dtype=torch.int32, device=DEV)
    free[:pages - len(rows)] = order[len(rows):]
    return {"case": case, "new": _ints(n), "lens": _ints(old), "table": table, "free": free, "count": _ints([pages - len(rows)]),
            "T": sum(max(a, 0) for a in n) + case["pad"], "count_out": _ints([0])}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if case["kind"] == "chunk":
        return _prepare_chunk(case, seed, gen)
    if case["kind"] == "plan":
        return _prepare_plan(case, seed, gen)
    s = {"case": case, "axis": _pair_axis(case)}
    D, Hq, Hkv, T, P = case["D"], case["Hq"], case["Hkv"], case["T"], case["P"]
    # a projection's rows: values of about 1, tokens of unlike size, some with large channels
    rows = _normal(gen, (T, (Hq + 2 * Hkv) * D))
    rows *= torch.exp(0.5 * torch.randn((T, 1), generator=gen, device=DEV)).bfloat16()
    rows[:, 3::97] *= 8
    s["qkv"] = rows
    wt = torch.bfloat16 if case["weights"] == "bf16" else torch.float32
    s["qw"], s["kw"] = ((1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(wt) for _ in range(2))
    half = case["R"] // 2
    freq = 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = torch.arange(P, device=DEV, dtype=torch.float64)[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    s["pos"] = torch.randint(0, P, (case["axes"], T), generator=gen, device=DEV, dtype=torch.int32)
    if case["kind"] == "axes_bwd":
        S = case["S"]
        shape = (lambda h: (T // S, h, S, D)) if S else (lambda h: (T, h, D))
        s["dq"], s["dk"], s["dv"] = (_normal(gen, shape(h), 0.01) for h in (Hq, Hkv, Hkv))
    if case["kind"] == "axes_cache":
        page = case["page"]
        pages = _pages(T, page) + 4
        shape = (pages, page, Hkv, D) if case["layout"] == "nhd" else (pages, Hkv, page, D)
        s["k_cache"], s["v_cache"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV), torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        s["slots"] = torch.randperm(pages * page, generator=gen, device=DEV)[:T].to(torch.int32)
        s["slots"][T - T // 16:] = -1  # padding of the step: its tokens are not written
    return s


# ------------------------------------------------------------------ the plain form
def _plain_chunk(s):
    """Request by request (its lengths are known to the program), kv head by kv head where the scores are many."""
    c = s["case"]
    Hq, Hkv, D, page, nhd = c["Hq"], c["Hkv"], c["D"], c["page"], c["layout"] == "nhd"
    G = Hq // Hkv
    o = torch.empty_like(s["q"])
    lse = torch.empty((Hq, o.shape[0]), device=DEV) if c["lse"] else None
    at = 0
    for b, (nq, nk) in enumerate(zip(s["ql"], s["kl"])):
        if not nq:
            continue
        rows = s["table"][b, :_pages(nk, page)].long()
        # [Hkv, nk, D] in 32 bits
        k, v = ((x[rows] if nhd else x[rows].transpose(1, 2)).reshape(-1, Hkv, D)[:nk].transpose(0, 1).float()
                for x in (s["k_cache"], s["v_cache"]))
        q = s["q"][at:at + nq].float().transpose(0, 1).reshape(Hkv, G * nq, D)
        hidden = None
        if c["causal"] and nq > 1:
            hidden = torch.arange(nk, device=DEV) > torch.arange(nq, device=DEV)[:, None] + (nk - nq)
        step = Hkv if nq * nk * Hq < 1 << 28 else 1
        for h in range(0, Hkv, step):
            p = (q[h:h + step] @ k[h:h + step].transpose(1, 2)).mul_(D ** -0.5).view(step * G, nq, nk)
            if hidden is not None:
                p.masked_fill_(hidden, -math.inf)
            m = p.amax(-1, keepdim=True)
            p = p.sub_(m).exp_()
            total = p.sum(-1, keepdim=True)
            out = (p.view(step, G * nq, nk) @ v[h:h + step]).view(step * G, nq, D) / total
            o[at:at + nq, h * G:(h + step) * G] = out.transpose(0, 1).bfloat16()
            if lse is not None:
                lse[h * G:(h + step) * G, at:at + nq] = (m + total.log())[..., 0]
        at += nq
    return (o, lse) if c["lse"] else (o,)


def _plain_plan(s):
    """The table is updated in place; a step can be planned again from the same lengths and list."""
    c = s["case"]
    page, T, table, free = c["page"], s["T"], s["table"], s["free"]
    new, old, F = s["new"].long(), s["lens"].long(), s["count"].long()
    B, most = table.shape
    over, n = new < 0, new.clamp(min=0)
    held = (old + page - 1) // page
    end = n.cumsum(0)
    cu = torch.cat((end.new_zeros(1), end)).clamp(max=T)
    fits = (old + n <= most * page) & (end <= T) & ~over
    need = torch.where(fits & (n > 0), (old + n + page - 1) // page - held, 0)
    off = need.cumsum(0) - need
    gives = torch.where(over, held, 0)
    given = gives.cumsum(0)
    total = (F + given[-1]).clamp(max=len(free))
    granted = fits & ((need == 0) | (off + need <= total))
    need = torch.where(granted, need, 0)
    taken = need.sum()
    j = torch.arange(most, device=DEV)
    # the list with the pages given back at its end
    back = table[over[:, None] & (j < held[:, None])]
    whole = torch.cat((free, torch.zeros_like(free)))
    at = F + torch.arange(len(back), device=DEV)
    whole[at] = back
    k = off[:, None] + j - held[:, None]
    fresh = (j >= held[:, None]) & (j < (held + need)[:, None])
    table.copy_(torch.where(fresh, whole[(total - 1 - k).clamp(0, len(whole) - 1)], table))
    left = total - taken
    index = torch.arange(len(free), device=DEV)
    free.copy_(torch.where((index >= F) & (index < left), whole[:len(free)], free))
    s["count_out"].copy_(left)
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(end, t, right=True).clamp(max=B - 1)
    here = (t < end[-1]) & granted[b]
    p = torch.where(here, old[b] + t - (end - n)[b], 0)
    at = table[b, (p // page).clamp(max=most - 1)].long()
    slots = torch.where(here & (at >= 0) & (at < len(free)), at * page + p % page, -1)
    lens = torch.where(over, 0, torch.where(granted, old + n, old))
    i32 = torch.int32
    return cu.to(i32), lens.to(i32), p.to(i32), slots.to(i32), torch.where(granted, n, 0).to(i32), table, free, s["count_out"]


def _turn(z, cos, sin, R, interleaved):
    """The rotation of the first R values of the last axis; cos and sin end in R / 2."""
    a, rest = z[..., :R], z[..., R:]
    if interleaved:
        x, y = a[..., 0::2], a[..., 1::2]
        return torch.cat((torch.stack((x * cos - y * sin, y * cos + x * sin), -1).flatten(-2), rest), -1)
    x, y = a[..., : R // 2], a[..., R // 2:]
    return torch.cat((x * cos - y * sin, y * cos + x * sin, rest), -1)


def _laid(x, S):
    """[T, H, D], or with S [T / S, H, S, D], in bf16 and contiguous."""
    x = x.bfloat16()
    return x.view(-1, S, *x.shape[1:]).transpose(1, 2).contiguous() if S else x.contiguous()


def _tokens(x, S):
    """The inverse of _laid, in 32 bits."""
    return (x.transpose(1, 2).reshape(-1, x.shape[1], x.shape[3]) if S else x).float()


def _rows(s):
    """The projection's q, k and v heads in 32 bits, and each token's angles, pair by pair from its axis' row."""
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    x = s["qkv"].float().view(c["T"], Hq + 2 * Hkv, c["D"])
    row = s["pos"].long()[list(s["axis"])].T  # [T, R / 2]
    pair = torch.arange(c["R"] // 2, device=DEV)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], s["cos"][row, pair][:, None], s["sin"][row, pair][:, None]


def _plain_axes_bwd_part(dy, x, w, cos, sin, c):
    g = _turn(dy, cos, -sin, c["R"], c["interleaved"])
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * r
    u = g * w.float()
    return r * (u - n * (u * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


def _plain_axes(s):
    c = s["case"]
    xq, xk, xv, cos, sin = _rows(s)
    if c["kind"] == "axes_bwd":
        dxq, dwq = _plain_axes_bwd_part(_tokens(s["dq"], c["S"]), xq, s["qw"], cos, sin, c)
        dxk, dwk = _plain_axes_bwd_part(_tokens(s["dk"], c["S"]), xk, s["kw"], cos, sin, c)
        return torch.cat((dxq, dxk, _tokens(s["dv"], c["S"])), 1).bfloat16().view(c["T"], -1), dwq, dwk
    q, k = (_turn(x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * w.float(), cos, sin, c["R"], c["interleaved"])
            for x, w in ((xq, s["qw"]), (xk, s["kw"])))
    if c["kind"] == "axes":
        return _laid(q, c["S"]), _laid(k, c["S"]), _laid(xv, c["S"])
    page, slots = c["page"], s["slots"].long()
    written = slots >= 0
    at, row = slots[written] // page, slots[written] % page
    for cache, x in ((s["k_cache"], k), (s["v_cache"], xv)):
        (cache if c["layout"] == "nhd" else cache.transpose(1, 2))[at, row] = x[written].bfloat16()
    return q.bfloat16(), s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    return (_plain_chunk if kind == "chunk" else _plain_plan if kind == "plan" else _plain_axes)(state)


def _run_own(s):
    import paper_2609_29219_gb300 as loom
    c = s["case"]
    kind = c["kind"]
    if kind == "chunk":
        r = loom.loom_attn_chunk_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["cu_q"], s["lens"], causal=c["causal"],
                                       layout=c["layout"], return_lse=c["lse"])
        return r if c["lse"] else (r,)
    if kind == "plan":
        out = loom.loom_paged_plan(s["new"], s["lens"], s["table"], s["free"], s["count"], s["T"], c["page"],
                                   free_count_out=s["count_out"])
        return (*out, s["table"], s["free"], s["count_out"])
    if kind == "axes":
        return loom.loom_qkv_norm_rope(s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], c["Hq"], c["Hkv"], s["pos"],
                                       seq_len=c["S"], eps=EPS, interleaved=c["interleaved"], pair_axis=s["axis"])
    if kind == "axes_bwd":
        return loom.loom_qkv_norm_rope_bwd(s["dq"], s["dk"], s["dv"], s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], s["pos"],
                                           eps=EPS, interleaved=c["interleaved"], pair_axis=s["axis"])
    q = loom.loom_qkv_norm_rope_cache(s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], s["pos"], s["slots"], s["k_cache"],
                                      s["v_cache"], c["Hq"], layout=c["layout"], eps=EPS, interleaved=c["interleaved"],
                                      pair_axis=s["axis"])
    return q, s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------ the same in 64 bits
def _exact_chunk(s):
    c = s["case"]
    Hq, Hkv, D, page = c["Hq"], c["Hkv"], c["D"], c["page"]
    g = Hq // Hkv
    offs = s["cu_q"].tolist()
    lens, table = s["lens"].tolist(), s["table"].tolist()
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros((Hq, o.shape[0]), dtype=torch.float64, device=DEV)
    for b, (first, last) in enumerate(zip(offs, offs[1:])):
        if first == last:
            continue
        n = lens[b]
        t = torch.arange(n, device=DEV)
        pages = torch.tensor(table[b], device=DEV)[torch.div(t, page, rounding_mode="floor")]
        for h in range(Hkv):
            if c["layout"] == "nhd":
                k, v = s["k_cache"][pages, t % page, h].double(), s["v_cache"][pages, t % page, h].double()
            else:
                k, v = s["k_cache"][pages, h, t % page].double(), s["v_cache"][pages, h, t % page].double()
            step = max(1, (1 << 27) // (g * n))
            for a in range(first, last, step):
                e = min(a + step, last)
                x = torch.einsum("igd,jd->igj", s["q"][a:e, h * g:(h + 1) * g].double(), k) / math.sqrt(D)
                if c["causal"]:
                    limit = torch.arange(a - last, e - last, device=DEV) + n  # the last key that each query sees
                    x = torch.where(t > limit[:, None, None], torch.full((), -math.inf, dtype=x.dtype, device=DEV), x)
                z = torch.logsumexp(x, -1)
                o[a:e, h * g:(h + 1) * g] = torch.einsum("igj,jd->igd", torch.exp(x - z[..., None]), v)
                lse[h * g:(h + 1) * g, a:e] = z.T
    return (o, lse) if c["lse"] else (o,)


def _exact_plan(s):
    """Request by request in Python's whole numbers."""
    page, T = s["case"]["page"], s["T"]
    new, old, table, free = s["new"].tolist(), s["lens"].tolist(), s["table"].tolist(), s["free"].tolist()
    stack = free[:int(s["count"])]
    for b, n in enumerate(new):
        if n < 0:
            stack += table[b][:_pages(old[b], page)]
    F = int(s["count"])
    room = len(stack)
    demand, cu, lens, granted, pos, slots = 0, [0], [], [], [0] * T, [-1] * T
    for b, n in enumerate(new):
        first = cu[-1]
        cu.append(first + max(n, 0))
        if n < 0 or old[b] + n > len(table[b]) * page or cu[-1] > T:
            lens.append(0 if n < 0 else old[b])
            granted.append(0)
            continue
        held = _pages(old[b], page)
        need = _pages(old[b] + n, page) - held if n else 0
        demand += need
        if need and demand > room:
            lens.append(old[b])
            granted.append(0)
            continue
        for j in range(need):
            table[b][held + j] = stack.pop()
        lens.append(old[b] + n)
        granted.append(n)
        for i in range(n):
            p = old[b] + i
            pos[first + i] = p
            slots[first + i] = table[b][p // page] * page + p % page
    for i in range(F, len(stack)):
        free[i] = stack[i]
    return tuple(_ints(x) for x in ([min(x, T) for x in cu], lens, pos, slots, granted, table, free, [len(stack)]))


def _exact_axes(s):
    c = s["case"]
    T, Hq, Hkv, D, R, S = c["T"], c["Hq"], c["Hkv"], c["D"], c["R"], c["S"]
    x = s["qkv"].double().reshape(T, -1, D)
    # over the whole head: y_i = z_i cos_i + sign_i z_partner(i) sin_i (values past R turn by nothing)
    cos, sin = torch.ones((T, D), dtype=torch.float64, device=DEV), torch.zeros((T, D), dtype=torch.float64, device=DEV)
    partner, sign = list(range(D)), [0.0] * D
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
        partner[a], partner[b], sign[a], sign[b] = b, a, -1.0, 1.0
        at = s["pos"][s["axis"][i]].long()
        cos[:, a] = cos[:, b] = s["cos"][at, i].double()
        sin[:, a] = sin[:, b] = s["sin"][at, i].double()
    cos, sin = cos[:, None], sin[:, None]
    partner, sign = torch.tensor(partner, device=DEV), torch.tensor(sign, dtype=torch.float64, device=DEV)
    w = torch.cat((s["qw"].double().expand(Hq, D), s["kw"].double().expand(Hkv, D)))
    xn = x[:, :Hq + Hkv]
    r = 1 / torch.sqrt((xn ** 2).sum(-1, keepdim=True) / D + EPS)
    if c["kind"] == "axes_bwd":
        back = (lambda t: t.double().permute(0, 2, 1, 3).reshape(T, -1, D)) if S else (lambda t: t.double())
        dy = torch.cat((back(s["dq"]), back(s["dk"])), 1)
        gz = dy * cos + (dy * sign * sin)[..., partner]  # the transpose of the forward's sum over partners
        n = xn * r
        dwh = (gz * n).sum(0)
        u = gz * w
        dx = (u - n * ((u * n).sum(-1, keepdim=True) / D)) * r
        return torch.cat((dx, back(s["dv"])), 1).reshape(T, -1), dwh[:Hq].sum(0), dwh[Hq:].sum(0)
    z = xn * r * w
    y = z * cos + sign * z[..., partner] * sin
    parts = y[:, :Hq], y[:, Hq:], x[:, Hq + Hkv:]
    if c["kind"] == "axes":
        return tuple(p.reshape(-1, S, p.shape[1], D).permute(0, 2, 1, 3).contiguous() if S else p.contiguous() for p in parts)
    caches = []
    for p in parts[1:]:
        cache = torch.zeros(s["k_cache"].shape, dtype=torch.float64, device=DEV)
        rows = cache if c["layout"] == "nhd" else cache.transpose(1, 2)
        keep = (s["slots"] >= 0).nonzero()[:, 0]
        slot = s["slots"][keep].long()
        rows[torch.div(slot, c["page"], rounding_mode="floor"), slot % c["page"]] = p[keep]
        caches.append(cache)
    return parts[0].contiguous(), caches[0], caches[1]


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_chunk if case["kind"] == "chunk" else _exact_plan if case["kind"] == "plan" else _exact_axes)(s)
