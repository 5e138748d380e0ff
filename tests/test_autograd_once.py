"""The autograd functions with torch stand-ins for the library's calls (no GPU needed): what they
return as gradients, and that what they have no gradient of is refused."""
import types

import pytest
import torch

from tests import grad_ref as ref


def _fwd(q, k, v, *, causal, scale, return_lse):
    o, lse = zip(*(ref.attention(*x, causal, scale) for x in zip(q, k, v)))
    return torch.stack(o), torch.stack(lse)


def _bwd(do, q, k, v, o, lse, *, causal, scale, dlse):
    none = [None] * len(q)
    grads = [ref.attention_grads(*x, causal, scale)[0] for x in zip(do, q, k, v, o, lse, none if dlse is None else dlse)]
    return tuple(map(torch.stack, zip(*grads)))


def _fwd_varlen(q, k, v, cu_q, cu_k, max_q, *, causal, scale, return_lse):
    o, lse = ref.attention(*(t.transpose(0, 1) for t in (q, k, v)), causal, scale)
    return o.transpose(0, 1).contiguous(), lse


def _bwd_varlen(do, q, k, v, o, lse, cu_q, cu_k, max_q, max_k, *, causal, scale, dlse):
    grads = ref.attention_grads(*(t.transpose(0, 1) for t in (do, q, k, v, o)), lse, dlse, causal, scale)[0]
    return tuple(g.transpose(0, 1).contiguous() for g in grads)


def _split(qkv, Hq, Hkv, D):
    return qkv.view(len(qkv), -1, D).split((Hq, Hkv, Hkv), 1)


def _norm(qkv, qw, kw, cos, sin, Hq, Hkv, positions, *, seq_len, eps, interleaved):
    q, k, v = _split(qkv, Hq, Hkv, len(qw))
    R = 2 * cos.shape[1]
    return (ref.norm_rope(q, qw, cos, sin, R, interleaved, eps), ref.norm_rope(k, kw, cos, sin, R, interleaved, eps), v.clone())


def _norm_bwd(dq, dk, dv, qkv, qw, kw, cos, sin, positions, *, eps, interleaved):
    q, k, _ = _split(qkv, dq.shape[1], dk.shape[1], len(qw))
    R = 2 * cos.shape[1]
    (dx, dqw), _ = ref.norm_rope_grads(dq, q, qw, cos, sin, R, interleaved, eps)
    (dy, dkw), _ = ref.norm_rope_grads(dk, k, kw, cos, sin, R, interleaved, eps)
    return torch.cat((dx, dy, dv), 1).flatten(1), dqw, dkw


@pytest.fixture
def autograd(monkeypatch):
    from paper_2609_29219_gb300 import autograd as module
    monkeypatch.setattr(module, "loom", types.SimpleNamespace(
        loom_attn_fwd=_fwd, loom_attn_bwd=_bwd, loom_attn_fwd_varlen=_fwd_varlen, loom_attn_bwd_varlen=_bwd_varlen,
        loom_qkv_norm_rope=_norm, loom_qkv_norm_rope_bwd=_norm_bwd,
        loom_gemm_bf16=lambda a, b, b_transposed=False: a @ (b.t() if b_transposed else b)))
    return module


def _rand(*shape, grad=True):
    return torch.randn(shape, generator=torch.Generator().manual_seed(sum(shape)), dtype=torch.float64).requires_grad_(grad)


def _calls(module):
    """(f, its differentiable arguments) of each function; f returns one tensor."""
    cu = torch.tensor([0, 5], dtype=torch.int32)
    angle = _rand(6, 4, grad=False)
    cat = lambda outs: torch.cat([t.flatten() for t in outs])  # noqa: E731
    return [
        (lambda *a: cat(module.attention(*a, causal=True, scale=0.3)), (_rand(2, 4, 5, 8), _rand(2, 2, 7, 8), _rand(2, 2, 7, 8))),
        (lambda *a: cat(module.attention_varlen(*a, cu, cu, 5, 5, scale=0.3)), (_rand(5, 4, 8), _rand(5, 2, 8), _rand(5, 2, 8))),
        (lambda *a: cat(module.qkv_norm_rope(*a, angle.cos(), angle.sin(), 2, 1, eps=0.1)), (_rand(6, 32), _rand(8), _rand(8))),
        (lambda *a: module.linear(*a), (_rand(4, 8), _rand(16, 8)))]


@pytest.mark.parametrize("i", range(4))
def test_first_gradients(autograd, i):
    """Against differences; with create_graph the values are the same."""
    f, args = _calls(autograd)[i]
    assert torch.autograd.gradcheck(f, args, eps=1e-6, atol=1e-7)
    plain = torch.autograd.grad(f(*args).square().sum(), args)
    kept = torch.autograd.grad(f(*args).square().sum(), args, create_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(plain, kept))


@pytest.mark.parametrize("i", range(4))
def test_a_second_differentiation_is_refused(autograd, i):
    """The kernels have first gradients only: a gradient's own gradient raises, it is not left out."""
    f, args = _calls(autograd)[i]
    out = f(*args)
    first = torch.autograd.grad(out.square().sum(), args[0], create_graph=True)[0]
    with pytest.raises(RuntimeError):
        (out.sum() + first.square().sum()).backward()


@pytest.mark.parametrize("which", ["cos", "sin"])
def test_tables_that_want_a_gradient_are_refused(autograd, which):
    tables = {n: _rand(6, 4, grad=n == which) for n in ("cos", "sin")}
    args = (_rand(6, 32), _rand(8), _rand(8), tables["cos"], tables["sin"], 2, 1)
    with pytest.raises(ValueError, match=which):
        autograd.qkv_norm_rope(*args)
    with torch.no_grad():  # nothing is differentiated here
        assert autograd.qkv_norm_rope(*args)[0].shape == (6, 2, 8)
