"""The library's attention and its QKV norm and rotation as torch autograd functions, for training.

    q, k, v = autograd.qkv_norm_rope(qkv, q_weight, k_weight, cos, sin, Hq, Hkv, seq_len=S)
    o, lse = autograd.attention(q, k, v, causal=True)

Each function saves its inputs (attention also O and LSE) and calls the entry points of the
package; a gradient of LSE is taken into account.  ``linear`` is the BF16 GEMM with its gradients.
The kernels have first gradients only: differentiating a gradient raises.
"""
from __future__ import annotations

import operator

import torch
from torch.autograd.function import once_differentiable

import paper_2609_29219_gb300 as loom


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, scale):
        o, lse = loom.loom_attn_fwd(q, k, v, causal=causal, scale=scale, return_lse=True)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.causal, ctx.scale = causal, scale
        ctx.set_materialize_grads(False)
        return o, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dlse):
        q, k, v, o, lse = ctx.saved_tensors
        do = torch.zeros_like(o) if do is None else do.contiguous()
        grads = loom.loom_attn_bwd(do, q, k, v, o, lse, causal=ctx.causal, scale=ctx.scale,
                                   dlse=None if dlse is None else dlse.contiguous())
        return (*grads, None, None)


def attention(q, k, v, *, causal=False, scale=None):
    """``loom_attn_fwd`` with gradients: (o, lse) of q [B,Hq,Sq,D], k and v [B,Hkv,Skv,D]."""
    return _Attention.apply(q, k, v, bool(causal), scale)


class _AttentionVarlen(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, max_q, max_k, causal, scale):
        o, lse = loom.loom_attn_fwd_varlen(q, k, v, cu_q, cu_k, max_q, causal=causal, scale=scale, return_lse=True)
        ctx.save_for_backward(q, k, v, o, lse, cu_q, cu_k)
        ctx.rest = (max_q, max_k, causal, scale)
        ctx.set_materialize_grads(False)
        return o, lse

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dlse):
        q, k, v, o, lse, cu_q, cu_k = ctx.saved_tensors
        max_q, max_k, causal, scale = ctx.rest
        do = torch.zeros_like(o) if do is None else do.contiguous()
        grads = loom.loom_attn_bwd_varlen(do, q, k, v, o, lse, cu_q, cu_k, max_q, max_k, causal=causal, scale=scale,
                                          dlse=None if dlse is None else dlse.contiguous())
        return (*grads, *(None,) * 6)


def attention_varlen(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, *, causal=False, scale=None):
    """``loom_attn_fwd_varlen`` with gradients: (o, lse) of packed tokens."""
    return _AttentionVarlen.apply(q, k, v, cu_seqlens_q, cu_seqlens_k, max_seqlen_q, max_seqlen_k, bool(causal), scale)


class _QkvNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions, seq_len, eps, interleaved, pair_axis):
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin, positions)
        ctx.shapes = (num_heads, num_kv_heads, seq_len)
        ctx.rest = {"eps": eps, "interleaved": interleaved, **({} if pair_axis is None else {"pair_axis": pair_axis})}
        return loom.loom_qkv_norm_rope(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions, seq_len=seq_len,
                                       **ctx.rest)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, q_weight, k_weight, cos, sin, positions = ctx.saved_tensors
        dqkv, dqw, dkw = loom.loom_qkv_norm_rope_bwd(dq.contiguous(), dk.contiguous(), dv.contiguous(), qkv, q_weight, k_weight,
                                                     cos, sin, positions, **ctx.rest)
        return (dqkv, dqw.to(q_weight.dtype), dkw.to(k_weight.dtype), *(None,) * 9)


def qkv_norm_rope(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions=None, *, seq_len=0, eps=1e-6,
                  interleaved=False, pair_axis=None):
    """``loom_qkv_norm_rope`` with gradients of qkv and the two norm weights: (q, k, v).  The tables have none."""
    for t, name in ((cos, "cos"), (sin, "sin")):
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which qkv_norm_rope does not have: detach it")
    return _QkvNormRope.apply(qkv, q_weight, k_weight, cos, sin, num_heads, num_kv_heads, positions, seq_len, eps, interleaved,
                              None if pair_axis is None else tuple(map(operator.index, pair_axis)))


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        ctx.save_for_backward(x, weight)
        return loom.loom_gemm_bf16(x, weight, b_transposed=True)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        dy = dy.contiguous()
        return loom.loom_gemm_bf16(dy, weight), loom.loom_gemm_bf16(dy.t().contiguous(), x)


def linear(x, weight):
    """x [T, K] times weight [N, K] transposed, by the BF16 GEMM, with gradients (T, N and K multiples of 8)."""
    return _Linear.apply(x, weight)
