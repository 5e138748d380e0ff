"""Cases of the operators around attention in training and serving: attention's backward pass,
and the norms of queries and keys with the position rotation.

A case is a dict of plain values.  ``kind`` names the operator:

* ``attn_bwd``         gradients of dense attention ([B, H, S, D]) from dO, Q, K, V, O and LSE
* ``attn_bwd_varlen``  the same over a ragged batch of packed tokens ([total, H, D])
* ``norm_rope``        a packed QKV projection to q, k (RMS norm per head, rotation) and v
* ``norm_rope_bwd``    its gradients: the projection's and the two norm weights'
* ``norm_rope_cache``  its serving form: k and v go to their slots of a cache

Sequence lengths of a ragged batch are a fixed set for a case (evenly spaced from ``lo`` to
``hi``, keys from ``klo`` to ``khi``), so that its work does not depend on the seed, which only
orders them.
"""
import math
import random

import torch

own = False  # True: run() calls the library; False: elementary torch operations in 32 bits

DEV = "cuda"
EPS = 1e-6


# ------------------------------------------------------------------ the cases
def _bwd(B, Hq, Hkv, Sq, Skv, D, causal, dlse=False):
    return {"kind": "attn_bwd", "B": B, "Hq": Hq, "Hkv": Hkv, "Sq": Sq, "Skv": Skv, "D": D, "causal": causal, "dlse": dlse}


def _bwd_varlen(B, Hq, Hkv, lo, hi, D, causal, klo=-1, khi=-1, dlse=False):
    """klo = -1: every sequence has as many keys as queries."""
    return {"kind": "attn_bwd_varlen", "B": B, "Hq": Hq, "Hkv": Hkv, "lo": lo, "hi": hi, "klo": klo, "khi": khi, "D": D,
            "causal": causal, "dlse": dlse}


def _rope(kind, T, Hq, Hkv, D, R, S, interleaved, weights, extra, P):
    """T tokens; S > 0: T / S sequences of S tokens, q, k, v [B, H, S, D]; S = 0: packed tokens with
    positions given, q, k, v [T, H, D].  extra: columns of the projection's rows after q, k, v.
    P: positions that the tables have."""
    return {"kind": kind, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "R": R, "S": S, "interleaved": interleaved, "weights": weights,
            "extra": extra, "P": P}


def _cache(T, Hq, Hkv, D, R, page, layout, interleaved, weights, extra, P):
    c = _rope("norm_rope_cache", T, Hq, Hkv, D, R, 0, interleaved, weights, extra, P)
    return dict(c, page=page, layout=layout)


def listed():
    named = [
        # the smallest backward pass: two heads, one tile of queries and keys; the launches are what costs
        ("bwd_tiny", _bwd(1, 2, 2, 128, 128, 64, False)),
        # a training step's batch in a decoder with a kv head for each query head
        ("bwd_b4_s2048_causal", _bwd(4, 32, 32, 2048, 2048, 128, True)),
        # one long sequence in a decoder with grouped queries; the largest case
        ("bwd_s8192_causal", _bwd(1, 32, 8, 8192, 8192, 128, True)),
        # training on a continuation: odd sizes, more keys than queries, a loss on the log-sum-exp too
        ("bwd_chunk_515_of_3001", _bwd(1, 32, 8, 515, 3001, 128, True, dlse=True)),
        # a step's documents of all lengths, packed without padding
        ("bwd_varlen_8_seqs", _bwd_varlen(8, 32, 8, 100, 2048, 128, True)),
        # short sequences against sequences of other lengths (cross attention), 64-wide heads
        ("bwd_varlen_cross_d64", _bwd_varlen(24, 16, 16, 17, 300, 64, False, klo=5, khi=700)),
        # the batch of the second case between its projection and its attention
        ("norm_rope_b4_s2048", _rope("norm_rope", 8192, 32, 8, 128, 128, 2048, False, "bf16", 0, 4096)),
        # a packed batch, half of each head rotated, interleaved pairs, a gate's columns in the same rows
        ("norm_rope_packed_odd", _rope("norm_rope", 3001, 16, 2, 64, 32, 0, True, "fp32", 24, 8192)),
        # the backward pass of both
        ("norm_rope_bwd_b4_s2048", _rope("norm_rope_bwd", 8192, 32, 8, 128, 128, 2048, False, "bf16", 0, 4096)),
        ("norm_rope_bwd_packed_odd", _rope("norm_rope_bwd", 1111, 16, 2, 64, 32, 0, True, "fp32", 24, 8192)),
        # one user's next token, into a paged cache: latency
        ("norm_rope_cache_one", _cache(1, 32, 8, 128, 128, 16, "nhd", False, "bf16", 0, 32768)),
        # a step of a busy server: next tokens and a prompt's chunk, padded, head-major pages
        ("norm_rope_cache_step", _cache(579, 32, 8, 128, 128, 64, "hnd", False, "bf16", 0, 32768)),
    ]
    return [dict(c, name=n) for n, c in named]


MOST_SCORES = 1.5e9  # a drawn case's most padded scores (the largest listed case has more)
MOST_VALUES = 4.0e7  # and the most values of a projection (the listed case has 5.0e7)


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over the logarithm."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


HEADS = ((32, 32), (32, 8), (64, 16), (16, 16), (16, 2), (8, 1), (8, 8), (6, 3))


def _draw_once(rng):
    kind = rng.choice(("attn_bwd", "attn_bwd", "attn_bwd_varlen", "attn_bwd_varlen", "norm_rope", "norm_rope_bwd", "norm_rope_cache"))
    D = rng.choice((64, 128))
    Hq, Hkv = rng.choice(HEADS)
    if kind == "attn_bwd":
        Sq = _log(rng, 1, 8192)
        Skv = Sq if rng.random() < 0.6 else _log(rng, Sq, 16384)
        if rng.random() < 0.1:
            Sq, Skv = Skv, Sq
        causal = rng.random() < 0.6 and Sq <= Skv
        # (where each query sees one key, dQ and dK are 0 without a gradient of LSE, and rounding noise is what remains)
        return _bwd(_log(rng, 1, 16), Hq, Hkv, Sq, Skv, D, causal, rng.random() < 0.3 or Skv < 4)
    if kind == "attn_bwd_varlen":
        hi = _log(rng, 2, 4096)
        lo = rng.choice((0, 1, _log(rng, 1, hi)))
        klo, khi = -1, -1
        if rng.random() < 0.35:
            khi = _log(rng, 2, 4096)
            klo = rng.choice((0, 1, _log(rng, 1, khi)))
        return _bwd_varlen(_log(rng, 2, 32), Hq, Hkv, lo, hi, D, rng.random() < 0.7, klo, khi,
                           rng.random() < 0.3 or hi < 4 or 0 <= khi < 4)
    R = rng.choice((D, D, D // 2, 16, 3 * D // 4))
    interleaved, weights = rng.random() < 0.4, rng.choice(("bf16", "bf16", "fp32"))
    extra, P = rng.choice((0, 0, 8, 8 * _log(rng, 1, 512))), _log(rng, 64, 32768)
    if kind == "norm_rope_cache":
        page = rng.choice((8, 16, 16, 32, 64, 192, 4096))
        return _cache(_log(rng, 1, 8192), Hq, Hkv, D, R, page, rng.choice(("nhd", "hnd")), interleaved, weights, extra, P)
    if rng.random() < 0.5:
        S = _log(rng, 1, 8192)
        return _rope(kind, S * _log(rng, 1, 8), Hq, Hkv, D, R, S, interleaved, weights, extra, max(P, S))
    return _rope(kind, _log(rng, 1, 32768), Hq, Hkv, D, R, 0, interleaved, weights, extra, P)


def draw(rng: random.Random):
    while True:
        c = _draw_once(rng)
        if c["kind"] == "attn_bwd":
            size = c["B"] * c["Hq"] * c["Sq"] * c["Skv"] / MOST_SCORES
        elif c["kind"] == "attn_bwd_varlen":
            size = c["B"] * c["Hq"] * c["hi"] * max(c["hi"] if c["klo"] < 0 else c["khi"], 1) / MOST_SCORES
        else:
            size = c["T"] * (c["D"] * (c["Hq"] + 2 * c["Hkv"]) + c["extra"]) / MOST_VALUES
        if size <= 1:
            return c


# ------------------------------------------------------------------ work
def _spaced(B, lo, hi):
    return [lo + round((hi - lo) * i / (B - 1)) for i in range(B)] if B > 1 else [hi]


def _dealt(case, seed):
    """The query and key lengths of a ragged batch's sequences: fixed pairs, in an order of the seed's."""
    ql = _spaced(case["B"], case["lo"], case["hi"])
    kl = list(ql) if case["klo"] < 0 else _spaced(case["B"], case["klo"], case["khi"])
    if case["klo"] >= 0:
        random.Random(1).shuffle(kl)
    both = list(zip(ql, kl))
    random.Random(seed).shuffle(both)
    return [a for a, _ in both], [b for _, b in both]


def _pairs(sq, skv, causal):
    """Visible (query, key) pairs: query i sees keys up to i + skv - sq."""
    if not causal:
        return sq * skv
    n = min(sq, skv)  # rows that see a key; the last sees skv
    return n * skv - n * (n - 1) // 2


def work(case):
    kind, D, Hq, Hkv = case["kind"], case["D"], case["Hq"], case["Hkv"]
    if kind in ("attn_bwd", "attn_bwd_varlen"):
        if kind == "attn_bwd":
            rows, keys = case["B"] * case["Sq"], case["B"] * case["Skv"]
            pairs = case["B"] * _pairs(case["Sq"], case["Skv"], case["causal"])
        else:
            ql, kl = _dealt(case, 0)
            rows, keys = sum(ql), sum(kl)
            pairs = sum(_pairs(a, b, case["causal"]) for a, b in zip(ql, kl))
        # read dO, Q, O, LSE, K, V; write dQ, dK, dV
        b = rows * Hq * (4 * 2 * D + 4) + keys * Hkv * 4 * 2 * D
        if case["dlse"]:
            b += rows * Hq * 4
        return {"bytes": b, "flops": 10 * D * Hq * pairs}
    T, R = case["T"], case["R"]
    normed, values = T * (Hq + Hkv) * D, T * (Hq + 2 * Hkv) * D
    wbytes = 2 * D * (2 if case["weights"] == "bf16" else 4)
    # a row of the tables for each position that occurs
    b = min(T, case["S"] or T, case["P"]) * R * 4 + wbytes + (0 if case["S"] else 4 * T)
    if kind == "norm_rope":
        return {"bytes": b + 2 * 2 * values, "flops": 9 * normed}
    if kind == "norm_rope_cache":
        return {"bytes": b + 4 * T + 2 * 2 * values, "flops": 9 * normed}
    # read dq, dk, dv and the projection's q and k parts; write its gradient and the weights'
    return {"bytes": b + 2 * (2 * values + normed) + 8 * D, "flops": 16 * normed}


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, std=1.0):
    t = torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)
    return t if std == 1.0 else t.mul_(std)


def _offsets(ls):
    offs = [0]
    for n in ls:
        offs.append(offs[-1] + n)
    return torch.tensor(offs, dtype=torch.int32, device=DEV)


def _tables(case):
    """cos, sin [P, R / 2] of the usual geometric frequencies."""
    half = case["R"] // 2
    freq = 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    angle = torch.arange(case["P"], device=DEV, dtype=torch.float64)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, s = case["kind"], {"case": case}
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    if kind == "attn_bwd":
        B, Sq, Skv = case["B"], case["Sq"], case["Skv"]
        s["q"], s["k"], s["v"] = (_normal(gen, (B, h, n, D)) for h, n in ((Hq, Sq), (Hkv, Skv), (Hkv, Skv)))
        s["do"] = _normal(gen, (B, Hq, Sq, D), 0.01)
        s["o"], s["lse"] = _forward(s["q"], s["k"], s["v"], _seen(Sq, Skv, case["causal"]))
        s["o"] = s["o"].bfloat16()
        s["dlse"] = 0.01 * torch.randn((B, Hq, Sq), generator=gen, device=DEV) if case["dlse"] else None
        return s
    if kind == "attn_bwd_varlen":
        ql, kl = _dealt(case, seed)
        tq, tk = sum(ql), sum(kl)
        s["cu_q"], s["cu_k"], s["max_q"], s["max_k"] = _offsets(ql), _offsets(kl), max(ql), max(kl)
        s["q"], s["k"], s["v"] = (_normal(gen, (n, h, D)) for h, n in ((Hq, tq), (Hkv, tk), (Hkv, tk)))
        s["do"] = _normal(gen, (tq, Hq, D), 0.01)
        q, k, v = _padded(s["q"], s["cu_q"], s["max_q"]), _padded(s["k"], s["cu_k"], s["max_k"]), _padded(s["v"], s["cu_k"], s["max_k"])
        o, lse = _forward(q, k, v, _seen_varlen(s["cu_q"], s["cu_k"], s["max_q"], s["max_k"], case["causal"]))
        s["o"] = _packed(o, s["cu_q"], tq).bfloat16()
        s["lse"] = _packed(lse[..., None], s["cu_q"], tq)[..., 0].T.contiguous()
        s["dlse"] = 0.01 * torch.randn((Hq, tq), generator=gen, device=DEV) if case["dlse"] else None
        return s
    T, P = case["T"], case["P"]
    width = (Hq + 2 * Hkv) * D
    # a projection's rows: values of about 1, tokens of unlike size, some with large channels
    rows = _normal(gen, (T, width + case["extra"]))
    rows *= torch.exp(0.5 * torch.randn((T, 1), generator=gen, device=DEV)).bfloat16()
    rows[:, 3::97] *= 8
    s["qkv"] = rows[:, :width]
    wt = torch.bfloat16 if case["weights"] == "bf16" else torch.float32
    s["qw"], s["kw"] = ((1 + 0.2 * torch.randn(D, generator=gen, device=DEV)).to(wt) for _ in range(2))
    s["cos"], s["sin"] = _tables(case)
    s["pos"] = None if case["S"] else torch.randint(0, P, (T,), generator=gen, device=DEV, dtype=torch.int32)
    if kind == "norm_rope_bwd":
        S = case["S"]
        shape = (lambda h: (T // S, h, S, D)) if S else (lambda h: (T, h, D))
        s["dq"], s["dk"], s["dv"] = (_normal(gen, shape(h), 0.01) for h in (Hq, Hkv, Hkv))
    if kind == "norm_rope_cache":
        page = case["page"]
        pages = -(-T // page) + 4
        shape = (pages, page, Hkv, D) if case["layout"] == "nhd" else (pages, Hkv, page, D)
        s["k_cache"], s["v_cache"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV), torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
        s["slots"] = torch.randperm(pages * page, generator=gen, device=DEV)[:T].to(torch.int32)
        s["slots"][T - T // 16:] = -1  # padding of the step: its tokens are not written
    return s


# ------------------------------------------------------------------ the plain form
def _seen(Sq, Skv, causal):
    """[Sq, Skv] of what each query sees, or None for everything."""
    if not causal:
        return None
    return torch.arange(Skv, device=DEV) <= torch.arange(Sq, device=DEV)[:, None] + (Skv - Sq)


def _seen_varlen(cu_q, cu_k, max_q, max_k, causal):
    """[B, 1, max_q, max_k] of what each query sees."""
    lq, lk = (c.diff().view(-1, 1, 1, 1) for c in (cu_q, cu_k))
    i, j = torch.arange(max_q, device=DEV)[:, None], torch.arange(max_k, device=DEV)
    seen = (i < lq) & (j < lk)
    return seen & (j <= i + (lk - lq)) if causal else seen


def _padded(x, cu, most):
    """Packed [total, H, D] as [B, H, most, D], zeros after each sequence's end."""
    at = torch.arange(most, device=DEV)
    inside = at < cu.diff()[:, None]
    if not x.shape[0]:
        return torch.zeros((len(cu) - 1, x.shape[1], most, x.shape[2]), dtype=x.dtype, device=DEV)
    rows = x[torch.where(inside, cu[:-1, None] + at, 0)]
    return (rows * inside[..., None, None]).transpose(1, 2)


def _packed(x, cu, total):
    """The inverse of _padded."""
    t = torch.arange(total, device=DEV, dtype=torch.int32)
    b = torch.searchsorted(cu, t, right=True) - 1
    return x[b, :, (t - cu[b])]


def _grouped(x, Hkv):
    """[B, Hq, S, D] as [B, Hkv, G * S, D]: the query heads of a kv head one after another."""
    B, Hq, S, D = x.shape
    return x.reshape(B, Hkv, Hq // Hkv * S, D)


def _scores(q, k, seen):
    """[B, Hkv, G, Sq, Skv] in 32 bits, -inf where a query does not see a key."""
    B, Hq, Sq, D = q.shape
    s = (_grouped(q, k.shape[1]) @ k.transpose(2, 3)).mul_(D ** -0.5).view(B, k.shape[1], -1, Sq, k.shape[2])
    if seen is not None:
        s.masked_fill_(~(seen.unsqueeze(2) if seen.dim() == 4 else seen), -math.inf)
    return s


def _forward(q, k, v, seen):
    """O [B, Hq, Sq, D] and LSE [B, Hq, Sq] in 32 bits; a query that sees nothing has 0 and -inf."""
    B, Hq, Sq, D = q.shape
    if not k.shape[2] or not Sq:
        return torch.zeros(q.shape, device=DEV), torch.full((B, Hq, Sq), -math.inf, device=DEV)
    s = _scores(q.float(), k.float(), seen)
    lse = s.logsumexp(-1)
    p = s.sub_(lse.clamp(min=-1e30)[..., None]).exp_()
    o = (p.view(B, k.shape[1], -1, k.shape[2]) @ v.float()).view(q.shape)
    return o, lse.view(B, Hq, Sq)


def _gradients(do, q, k, v, o, lse, dlse, seen):
    """dQ, dK, dV in 32 bits of padded or dense tensors."""
    B, Hq, Sq, D = q.shape
    Hkv, Skv = k.shape[1], k.shape[2]
    do, q, k, v, o = (x.float() for x in (do, q, k, v, o))
    p = _scores(q, k, seen).sub_(lse.clamp(min=-1e30).view(B, Hkv, -1, Sq, 1)).exp_().view(B, Hkv, -1, Skv)
    delta = (do * o).sum(-1)
    if dlse is not None:
        delta = delta - dlse
    qg, dog = _grouped(q, Hkv), _grouped(do, Hkv)
    dv = p.transpose(2, 3) @ dog
    ds = (dog @ v.transpose(2, 3)).sub_(delta.view(B, Hkv, -1, 1)).mul_(p).mul_(D ** -0.5)
    return (ds @ k).view(q.shape), ds.transpose(2, 3) @ qg, dv


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
    """The projection's q, k and v heads in 32 bits, and each token's row of the tables."""
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    x = s["qkv"].float().view(c["T"], Hq + 2 * Hkv, c["D"])
    pos = torch.arange(c["T"], device=DEV) % c["S"] if c["S"] else s["pos"].long()
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], s["cos"][pos][:, None], s["sin"][pos][:, None]


def _normed(x):
    return x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def _plain_rope(s):
    c = s["case"]
    xq, xk, xv, cos, sin = _rows(s)
    q = _turn(_normed(xq) * s["qw"].float(), cos, sin, c["R"], c["interleaved"])
    k = _turn(_normed(xk) * s["kw"].float(), cos, sin, c["R"], c["interleaved"])
    return q, k, xv


def _plain_rope_part_bwd(dy, x, w, cos, sin, c):
    g = _turn(dy, cos, -sin, c["R"], c["interleaved"])
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    n = x * r
    u = g * w.float()
    return r * (u - n * (u * n).mean(-1, keepdim=True)), (g * n).sum((0, 1))


# ------------------------------------------------------------------ one pass
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "attn_bwd":
        grads = _gradients(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["dlse"], _seen(c["Sq"], c["Skv"], c["causal"]))
        return tuple(g.bfloat16() for g in grads)
    if kind == "attn_bwd_varlen":
        cu_q, cu_k, max_q, max_k = s["cu_q"], s["cu_k"], s["max_q"], s["max_k"]
        tq, tk = s["q"].shape[0], s["k"].shape[0]
        do, q, o = (_padded(s[n], cu_q, max_q) for n in ("do", "q", "o"))
        k, v = (_padded(s[n], cu_k, max_k) for n in ("k", "v"))
        lse = _padded(s["lse"].T[..., None], cu_q, max_q)[..., 0]
        dlse = None if s["dlse"] is None else _padded(s["dlse"].T[..., None], cu_q, max_q)[..., 0]
        dq, dk, dv = _gradients(do, q, k, v, o, lse.nan_to_num(neginf=-1e30), dlse, _seen_varlen(cu_q, cu_k, max_q, max_k, c["causal"]))
        return _packed(dq.bfloat16(), cu_q, tq), _packed(dk.bfloat16(), cu_k, tk), _packed(dv.bfloat16(), cu_k, tk)
    if kind == "norm_rope_bwd":
        xq, xk, _, cos, sin = _rows(s)
        dxq, dwq = _plain_rope_part_bwd(_tokens(s["dq"], c["S"]), xq, s["qw"], cos, sin, c)
        dxk, dwk = _plain_rope_part_bwd(_tokens(s["dk"], c["S"]), xk, s["kw"], cos, sin, c)
        dqkv = torch.cat((dxq, dxk, _tokens(s["dv"], c["S"])), 1).bfloat16().view(c["T"], -1)
        return dqkv, dwq, dwk
    q, k, v = _plain_rope(s)
    if kind == "norm_rope":
        return _laid(q, c["S"]), _laid(k, c["S"]), _laid(v, c["S"])
    page, slots = c["page"], s["slots"].long()
    written = slots >= 0
    at, row = slots[written] // page, slots[written] % page
    for cache, x in ((s["k_cache"], k), (s["v_cache"], v)):
        (cache if c["layout"] == "nhd" else cache.transpose(1, 2))[at, row] = x[written].bfloat16()
    return q.bfloat16(), s["k_cache"], s["v_cache"]


def _run_own(s):
    import paper_2609_29219_gb300 as loom
    c = s["case"]
    kind = c["kind"]
    if kind == "attn_bwd":
        return loom.loom_attn_bwd(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], causal=c["causal"], dlse=s["dlse"])
    if kind == "attn_bwd_varlen":
        return loom.loom_attn_bwd_varlen(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["cu_q"], s["cu_k"], s["max_q"],
                                         s["max_k"], causal=c["causal"], dlse=s["dlse"])
    if kind == "norm_rope":
        return loom.loom_qkv_norm_rope(s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], c["Hq"], c["Hkv"], s["pos"],
                                       seq_len=c["S"], eps=EPS, interleaved=c["interleaved"])
    if kind == "norm_rope_bwd":
        return loom.loom_qkv_norm_rope_bwd(s["dq"], s["dk"], s["dv"], s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], s["pos"],
                                           eps=EPS, interleaved=c["interleaved"])
    q = loom.loom_qkv_norm_rope_cache(s["qkv"], s["qw"], s["kw"], s["cos"], s["sin"], s["pos"], s["slots"], s["k_cache"],
                                      s["v_cache"], c["Hq"], layout=c["layout"], eps=EPS, interleaved=c["interleaved"])
    return q, s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------ the same in 64 bits
def _exact_attend(do, q, k, v, o, lse, dlse, causal):
    """Gradients for one kv head, all float64: do, q, o [g, sq, D], lse [g, sq], k, v [skv, D]."""
    g, sq, D = q.shape
    skv = k.shape[0]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    delta = torch.einsum("gid,gid->gi", do, o)
    if dlse is not None:
        delta -= dlse
    step = max(1, (1 << 27) // max(1, g * skv))
    for a in range(0, sq, step):
        e = min(sq, a + step)
        n = max(0, min(skv, e + skv - sq)) if causal else skv  # keys that these queries may see
        if not n:
            continue
        p = torch.exp(torch.einsum("gid,jd->gij", q[:, a:e], k[:n]) / math.sqrt(D) - lse[:, a:e, None])
        if causal:
            last = torch.arange(a, e, device=DEV) + (skv - sq)
            p = torch.where(torch.arange(n, device=DEV) > last[:, None], torch.zeros((), dtype=p.dtype, device=DEV), p)
        dv[:n] += torch.einsum("gij,gid->jd", p, do[:, a:e])
        p *= (torch.einsum("gid,jd->gij", do[:, a:e], v[:n]) - delta[:, a:e, None]) / math.sqrt(D)
        dq[:, a:e] = torch.einsum("gij,jd->gid", p, k[:n])
        dk[:n] += torch.einsum("gij,gid->jd", p, q[:, a:e])
    return dq, dk, dv


def _exact_attn(s):
    c = s["case"]
    Hq, Hkv = c["Hq"], c["Hkv"]
    g = Hq // Hkv
    dq, dk, dv = (torch.zeros(s[n].shape, dtype=torch.float64, device=DEV) for n in "qkv")
    d = lambda x: x.double().contiguous()  # noqa: E731
    if c["kind"] == "attn_bwd":
        for b in range(c["B"]):
            for h in range(Hkv):
                hs = slice(h * g, (h + 1) * g)
                dq[b, hs], dk[b, h], dv[b, h] = _exact_attend(
                    d(s["do"][b, hs]), d(s["q"][b, hs]), d(s["k"][b, h]), d(s["v"][b, h]), d(s["o"][b, hs]), d(s["lse"][b, hs]),
                    None if s["dlse"] is None else d(s["dlse"][b, hs]), c["causal"])
        return dq, dk, dv
    oq, ok = s["cu_q"].tolist(), s["cu_k"].tolist()
    for qa, qe, ka, ke in zip(oq, oq[1:], ok, ok[1:]):
        for h in range(Hkv):
            hs = slice(h * g, (h + 1) * g)
            x, y, z = _exact_attend(
                d(s["do"][qa:qe, hs].transpose(0, 1)), d(s["q"][qa:qe, hs].transpose(0, 1)), d(s["k"][ka:ke, h]), d(s["v"][ka:ke, h]),
                d(s["o"][qa:qe, hs].transpose(0, 1)), d(s["lse"][hs, qa:qe]),
                None if s["dlse"] is None else d(s["dlse"][hs, qa:qe]), c["causal"])
            dq[qa:qe, hs], dk[ka:ke, h], dv[ka:ke, h] = x.transpose(0, 1), y, z
    return dq, dk, dv


def _exact_angles(s):
    """cos and sin of each token over the whole head, and the index and sign of each value's partner:
    y_i = z_i cos_i + sign_i z_partner(i) sin_i (values past R turn by nothing)."""
    c = s["case"]
    D, R = c["D"], c["R"]
    pos = torch.tensor([t % c["S"] for t in range(c["T"])], device=DEV) if c["S"] else s["pos"].long()
    cos, sin = torch.ones((c["T"], D), dtype=torch.float64, device=DEV), torch.zeros((c["T"], D), dtype=torch.float64, device=DEV)
    partner, sign = list(range(D)), [0.0] * D
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
        partner[a], partner[b], sign[a], sign[b] = b, a, -1.0, 1.0
        cos[:, a] = cos[:, b] = s["cos"][pos, i].double()
        sin[:, a] = sin[:, b] = s["sin"][pos, i].double()
    return cos[:, None], sin[:, None], torch.tensor(partner, device=DEV), torch.tensor(sign, dtype=torch.float64, device=DEV)


def _exact_rope(s):
    c = s["case"]
    T, Hq, Hkv, D, S = c["T"], c["Hq"], c["Hkv"], c["D"], c["S"]
    x = s["qkv"].double().reshape(T, -1, D)
    cos, sin, partner, sign = _exact_angles(s)
    w = torch.cat((s["qw"].double().expand(Hq, D), s["kw"].double().expand(Hkv, D)))
    xn = x[:, :Hq + Hkv]
    r = 1 / torch.sqrt((xn ** 2).sum(-1, keepdim=True) / D + EPS)
    if c["kind"] == "norm_rope_bwd":
        back = (lambda t: t.double().permute(0, 2, 1, 3).reshape(T, -1, D)) if S else (lambda t: t.double())
        dy = torch.cat((back(s["dq"]), back(s["dk"])), 1)
        # the transpose of the forward's sum over partners
        gz = dy * cos + (dy * sign * sin)[..., partner]
        n = xn * r
        dwh = (gz * n).sum(0)
        u = gz * w
        dx = (u - n * ((u * n).sum(-1, keepdim=True) / D)) * r
        return torch.cat((dx, back(s["dv"])), 1).reshape(T, -1), dwh[:Hq].sum(0), dwh[Hq:].sum(0)
    z = xn * r * w
    y = z * cos + sign * z[..., partner] * sin
    parts = y[:, :Hq], y[:, Hq:], x[:, Hq + Hkv:]
    if c["kind"] == "norm_rope":
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
    return _exact_attn(s) if case["kind"].startswith("attn") else _exact_rope(s)
