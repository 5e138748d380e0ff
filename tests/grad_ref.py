"""Attention's gradients and the norm-and-rotation operator in 64 bits, and how far a kernel that
rounds as the library says may be from them (no GPU needed).

Attention: the kernel holds scores, sums and gradients in fp32, rounds P and dS to bf16 (relative
2^-8 at most) before they meet dO, Q and K, and each gradient once more when it is stored.  So
    |dV - exact| <= 2^-8 |dV| + 2^-8 sum P |dO|            (and dQ, dK with |dS| |K|, |dS| |Q|)
plus what fp32 leaves: P is off by about 2^-21 + 2^-23 |s| relative (the exponent's products,
2^x and the statistics), dP and delta by 2^-21 of their sums of magnitudes.  FP32 below is 2^-17
of the magnitudes: 16 times that, so that an exponent of up to 30 is covered too.
"""
import torch

BF16 = 2.0 ** -8
FP32 = 2.0 ** -17


def seen_mask(sq, skv, causal):
    """[sq, skv]: query i sees key j (bottom-right aligned)."""
    if not causal:
        return torch.ones((sq, skv), dtype=torch.bool)
    return torch.arange(skv)[None, :] <= torch.arange(sq)[:, None] + (skv - sq)


def attention(q, k, v, causal, scale):
    """float64 O [Hq, sq, D] and LSE of one sequence: q [Hq, sq, D], k, v [Hkv, skv, D]."""
    G = q.shape[0] // k.shape[0]
    k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = scale * q @ k.transpose(1, 2)
    s = s.masked_fill(~seen_mask(q.shape[1], k.shape[1], causal), -float("inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    return p @ v, lse


def attention_grads(do, q, k, v, o, lse, dlse, causal, scale):
    """((dq, dk, dv), (their bounds)) of one sequence, float64 in and out."""
    Hkv, skv, D = k.shape
    Hq, sq, _ = q.shape
    G = Hq // Hkv
    ke, ve = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = scale * q @ ke.transpose(1, 2)
    s = s.masked_fill(~seen_mask(sq, skv, causal), -float("inf"))
    p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    delta = (do * o).sum(-1)
    mag = do.abs() @ ve.abs().transpose(1, 2) + (do * o).abs().sum(-1)[..., None]
    if dlse is not None:
        delta = delta - dlse
        mag = mag + dlse.abs()[..., None]
    ds = p * (do @ ve.transpose(1, 2) - delta[..., None]) * scale
    mag = p * mag * scale
    group = lambda x: x.view(Hkv, G, skv, D).sum(1)  # noqa: E731
    dq, dk, dv = ds @ ke, group(ds.transpose(1, 2) @ q), group(p.transpose(1, 2) @ do)
    bq = BF16 * (dq.abs() + ds.abs() @ ke.abs()) + FP32 * (mag @ ke.abs())
    bk = BF16 * (dk.abs() + group(ds.abs().transpose(1, 2) @ q.abs())) + FP32 * group(mag.transpose(1, 2) @ q.abs())
    bv = (BF16 + FP32) * group(p.transpose(1, 2) @ do.abs()) + BF16 * dv.abs()
    return (dq, dk, dv), tuple(1.01 * b + 1e-30 for b in (bq, bk, bv))


def rotate(z, cos, sin, R, interleaved):
    """z [T, H, D], cos and sin [T, R / 2], all float64."""
    out = z.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        c, s = cos[:, None, i], sin[:, None, i]
        out[..., a] = z[..., a] * c - z[..., b] * s
        out[..., b] = z[..., b] * c + z[..., a] * s
    return out


def norm_rope(x, w, cos, sin, R, interleaved, eps):
    """Norm and rotation of heads x [T, H, D] in float64."""
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return rotate(x * r * w, cos, sin, R, interleaved)


def norm_rope_grads(dy, x, w, cos, sin, R, interleaved, eps):
    """((dx, dw), (their bounds)): dx is rounded once to bf16, the rest is fp32."""
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    g = rotate(dy, cos, -sin, R, interleaved)
    n = x * r
    u = g * w
    dx = r * (u - n * (u * n).mean(-1, keepdim=True))
    dw = (g * n).sum((0, 1))
    mag = rotate(dy.abs(), cos.abs(), -sin.abs(), R, interleaved)  # (a bound of |g| for each half of a pair)
    mag = torch.maximum(mag.abs(), rotate(dy.abs(), cos.abs(), sin.abs(), R, interleaved).abs())
    mu = mag * w.abs()
    bx = BF16 * dx.abs() + FP32 * r * (mu + n.abs() * (mu * n.abs()).mean(-1, keepdim=True))
    return (dx, dw), (1.01 * bx + 1e-30, FP32 * (mag * n.abs()).sum((0, 1)) + 1e-30)
