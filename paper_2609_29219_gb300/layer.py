"""A decoder's attention layer on the library: trained with its gradients, then run over a paged cache
with the same weights, token by token, or with whatever tokens each request brings to a step.

    python -m paper_2609_29219_gb300.layer

trains a small layer for some steps to imitate another one, prints the loss, and checks that
decoding the sequence through the cache gives what the prefill gives, and that serving requests of
unlike lengths in chunks does.
"""
from __future__ import annotations

import torch

import paper_2609_29219_gb300 as loom
from paper_2609_29219_gb300 import autograd


def rope_tables(positions, rotary_dim, base=10000.0, device="cuda"):
    """cos and sin [positions, rotary_dim / 2] of the usual geometric frequencies."""
    half = rotary_dim // 2
    freq = base ** (-torch.arange(half, device=device, dtype=torch.float64) / half)
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


class PagedCache:
    """K and V pages [num_pages, page, Hkv, D] and the pages of each sequence, given out in order.
    Every sequence has `used` tokens (on the host; `lens` on the device) of `capacity`, whole pages."""

    def __init__(self, sequences, capacity, Hkv, D, page=16, device="cuda"):
        per = -(-capacity // page)
        self.page, self.device = page, device
        self.capacity, self.used = per * page, 0
        self.k, self.v = (torch.zeros((sequences * per, page, Hkv, D), dtype=torch.bfloat16, device=device) for _ in range(2))
        self.table = torch.randperm(sequences * per, device=device).to(torch.int32).view(sequences, per)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=device)

    def take(self, count):
        """Positions and slots of each sequence's next `count` tokens, token-major by sequence."""
        if not 0 <= count <= self.capacity - self.used:
            raise ValueError(f"the cache has room for {self.capacity - self.used} more tokens a sequence, not {count}")
        pos = self.lens[:, None] + torch.arange(count, dtype=torch.int32, device=self.device)
        slots = self.table.gather(1, (pos // self.page).long()) * self.page + pos % self.page
        self.lens += count
        self.used += count
        return pos.reshape(-1), slots.reshape(-1)


class RequestCache:
    """K and V pages [num_pages, page, Hkv, D] shared by up to `requests` requests of `capacity` tokens (whole
    pages), which take pages as they grow and give them back when they end.  All of it is on the device: a step
    that was captured can be replayed.  `granted`: the tokens of each request that the last step that a
    layer served had room for (all that it brought, or none)."""

    def __init__(self, requests, num_pages, capacity, Hkv, D, page=16, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.page, per = page, -(-capacity // page)
        self.capacity = per * page
        self.k, self.v = (torch.zeros((num_pages, page, Hkv, D), dtype=torch.bfloat16, device=device) for _ in range(2))
        self.table = torch.full((requests, per), -1, **i32)
        self.lens, self.granted = (torch.zeros(requests, **i32) for _ in range(2))
        self.free_pages, self.free_count = torch.arange(num_pages, **i32), torch.full((1,), num_pages, **i32)

    def plan(self, new_lens, num_tokens, granted=None):
        """Takes `new_lens` more tokens of each request (negative: it is over) into a step of num_tokens:
        (cu_seqlens, positions, slots, granted), the last one written to the tensor given or a new one."""
        cu, _, positions, slots, granted = loom.loom_paged_plan(new_lens, self.lens, self.table, self.free_pages, self.free_count,
                                                                num_tokens, self.page, seqlens_k=self.lens, granted=granted)
        return cu, positions, slots, granted


class AttentionLayer:
    """y = attention(rotated norms of x W_qkv^T) W_o^T with grouped queries; weights in bf16."""

    def __init__(self, model, Hq, Hkv, D, positions, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda n, k: (torch.randn((n, k), generator=gen, device=device) * k ** -0.5).bfloat16().requires_grad_()  # noqa: E731
        self.Hq, self.Hkv, self.D = Hq, Hkv, D
        self.w_qkv, self.w_o = new((Hq + 2 * Hkv) * D, model), new(model, Hq * D)
        self.q_norm, self.k_norm = (torch.ones(D, device=device, requires_grad=True) for _ in range(2))
        self.cos, self.sin = rope_tables(positions, D, device=device)

    def parameters(self):
        return [self.w_qkv, self.w_o, self.q_norm, self.k_norm]

    def forward(self, x):
        """x [B, S, model] with gradients (B S a multiple of 8)."""
        B, S, model = x.shape
        qkv = autograd.linear(x.reshape(B * S, model), self.w_qkv)
        q, k, v = autograd.qkv_norm_rope(qkv, self.q_norm, self.k_norm, self.cos, self.sin, self.Hq, self.Hkv, seq_len=S)
        o, _ = autograd.attention(q, k, v, causal=True)
        return autograd.linear(o.transpose(1, 2).reshape(B * S, -1), self.w_o).view(B, S, model)

    @torch.no_grad()
    def step(self, x, cache):
        """One token of each sequence, x [B, model]: its k and v go into the cache, its query reads it."""
        if cache.used >= self.cos.shape[0]:
            raise ValueError(f"the rotation tables have no position {cache.used}")
        pos, slots = cache.take(1)
        qkv = loom.loom_gemm_bf16(x, self.w_qkv, b_transposed=True)
        q = loom.loom_qkv_norm_rope_cache(qkv, self.q_norm, self.k_norm, self.cos, self.sin, pos, slots, cache.k, cache.v, self.Hq)
        o = loom.loom_attn_decode_paged(q.unsqueeze(2), cache.k, cache.v, cache.table, cache.lens)
        return loom.loom_gemm_bf16(o.view(x.shape[0], -1), self.w_o, b_transposed=True)

    @torch.no_grad()
    def serve(self, x, cache, new_lens):
        """The new tokens of a RequestCache's requests, packed, x [T, model]: prompts, chunks of them, single tokens.
        Rows past the last request's (and those of requests that the cache had no room for: cache.granted) mean
        nothing.  The rotation tables must reach the cache's capacity.  An x or a cache that is refused leaves the
        cache as it was.  (The step is planned here: a model of several layers plans once and makes the calls after
        that a layer.  Where each request brings one token the paged decode is mostly the faster call: see step.)"""
        if x.dim() != 2 or x.shape[1] != self.w_qkv.shape[1]:
            raise ValueError(f"x must be [T, model] with a model of {self.w_qkv.shape[1]}, got shape {tuple(x.shape)}")
        if tuple(cache.k.shape[2:]) != (self.Hkv, self.D):
            raise ValueError(f"the cache's heads are {tuple(cache.k.shape[2:])}, the layer's {(self.Hkv, self.D)}")
        if cache.capacity > self.cos.shape[0]:
            raise ValueError(f"the rotation tables have {self.cos.shape[0]} positions, the cache's requests up to {cache.capacity} tokens")
        if not x.shape[0]:
            cache.plan(new_lens, 0, cache.granted)
            return torch.empty_like(x)
        qkv = loom.loom_gemm_bf16(x, self.w_qkv, b_transposed=True)  # (it refuses what else x may be, before anything is taken)
        cu, positions, slots, _ = cache.plan(new_lens, x.shape[0], cache.granted)
        q = loom.loom_qkv_norm_rope_cache(qkv, self.q_norm, self.k_norm, self.cos, self.sin, positions, slots, cache.k, cache.v, self.Hq)
        o = loom.loom_attn_chunk_paged(q, cache.k, cache.v, cache.table, cu, cache.lens)
        return loom.loom_gemm_bf16(o.view(x.shape[0], -1), self.w_o, b_transposed=True)


def train(layer, teacher, steps, B=2, S=128, rate=5e-3, seed=1):
    """Losses of `steps` steps of Adam towards the teacher's outputs (moments and master weights in fp32)."""
    model = layer.w_qkv.shape[1]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    masters = [p.detach().float().clone().requires_grad_() for p in layer.parameters()]
    optimizer = torch.optim.Adam(masters, lr=rate, betas=(0.9, 0.95))
    losses = []
    for _ in range(steps):
        x = torch.randn((B, S, model), generator=gen, device="cuda").bfloat16()
        with torch.no_grad():
            want = teacher.forward(x).float()
        loss = (layer.forward(x).float() - want).square().mean()
        loss.backward()
        for p, m in zip(layer.parameters(), masters):
            m.grad, p.grad = p.grad.float(), None
        optimizer.step()
        with torch.no_grad():
            for p, m in zip(layer.parameters(), masters):
                p.copy_(m)
        losses.append(loss.item())
    return losses


def main():
    shape = dict(model=512, Hq=8, Hkv=2, D=64, positions=256)
    layer, teacher = AttentionLayer(**shape, seed=0), AttentionLayer(**shape, seed=7)
    losses = train(layer, teacher, 60)
    print("loss " + " ".join(f"{x:.4f}" for x in losses[::10] + losses[-1:]))
    B, S = 2, 40
    x = torch.randn((B, S, shape["model"]), device="cuda").bfloat16()
    with torch.no_grad():
        want = layer.forward(x)
    cache = PagedCache(B, S, shape["Hkv"], shape["D"])
    got = torch.stack([layer.step(x[:, i].contiguous(), cache) for i in range(S)], 1)
    loom.loom_attn_check_error()
    requests = RequestCache(B, 16, 64, shape["Hkv"], shape["D"])
    parts, done = [[] for _ in range(B)], [0] * B
    for new in ((17, 3), (1, 30), (22, 7)):
        y = layer.serve(torch.cat([x[b, done[b]:done[b] + n] for b, n in enumerate(new)]), requests,
                        torch.tensor(new, dtype=torch.int32, device="cuda"))
        for b, (n, part) in enumerate(zip(new, y.split(new))):
            parts[b].append(part)
            done[b] += n
    served = torch.stack([torch.cat(p) for p in parts])
    loom.loom_attn_check_error()
    print(f"serving in chunks against prefill: largest difference {float((served.float() - want.float()).abs().max()):.2e}")
    print(f"decoding token by token against prefill: largest difference {float((got.float() - want.float()).abs().max()):.2e} "
          f"of {float(want.float().abs().max()):.2f}")


if __name__ == "__main__":
    main()
