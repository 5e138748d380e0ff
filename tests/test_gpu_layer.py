"""The training and serving entry points together: a layer trained with their gradients, and its
decoding through the cache against its prefill."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layer_mod():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_29219_gb300 import layer
    return layer


def test_training_lowers_the_loss_and_decoding_matches_prefill(layer_mod):
    import torch

    import paper_2609_29219_gb300 as loom
    shape = dict(model=256, Hq=4, Hkv=2, D=64, positions=128)
    layer, teacher = layer_mod.AttentionLayer(**shape, seed=0), layer_mod.AttentionLayer(**shape, seed=7)
    losses = layer_mod.train(layer, teacher, 40)
    assert sum(losses[-5:]) < 0.7 * sum(losses[:5])
    x = torch.randn((3, 33, 256), device="cuda").bfloat16()[:, :32].contiguous()
    with torch.no_grad():
        want = layer.forward(x).float()
    cache = layer_mod.PagedCache(3, 32, 2, 64)
    got = torch.stack([layer.step(x[:, i].contiguous(), cache) for i in range(32)], 1).float()
    loom.loom_attn_check_error()
    # both round q, k, v, P, O and the result to bf16: a few units of 2^-8 of the largest value
    assert float((got - want).abs().max()) <= 2 ** -5 * float(want.abs().max())


def test_gradients_of_the_layer_against_torch(layer_mod):
    """All of the chain's gradients against torch's own in 64 bits."""
    import torch

    from tests import grad_ref as ref
    layer = layer_mod.AttentionLayer(model=128, Hq=4, Hkv=2, D=64, positions=64, seed=3)
    B, S = 2, 48
    x = torch.randn((B, S, 128), device="cuda").bfloat16()
    up = torch.randn((B, S, 128), device="cuda").bfloat16()
    layer.forward(x).backward(up)
    w_qkv, w_o, qn, kn = [p.detach().double().cpu().requires_grad_() for p in layer.parameters()]
    cos, sin = layer.cos[:S].double().cpu(), layer.sin[:S].double().cpu()
    rot = lambda z: torch.cat((z[..., :32] * cos[:, None] - z[..., 32:] * sin[:, None],  # noqa: E731
                               z[..., 32:] * cos[:, None] + z[..., :32] * sin[:, None]), -1)
    norm = lambda z, w: z / (z.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w  # noqa: E731
    total = 0
    for b in range(B):
        h = (x[b].double().cpu() @ w_qkv.T).view(S, 8, 64)
        q, k, v = rot(norm(h[:, :4], qn)), rot(norm(h[:, 4:6], kn)), h[:, 6:]
        o, _ = ref.attention(q.transpose(0, 1), k.transpose(0, 1), v.transpose(0, 1), True, 0.125)
        total = total + (o.transpose(0, 1).reshape(S, -1) @ w_o.T * up[b].double().cpu()).sum()
    total.backward()
    for p, r, n in zip(layer.parameters(), (w_qkv, w_o, qn, kn), ("w_qkv", "w_o", "q_norm", "k_norm")):
        got, want = p.grad.double().cpu(), r.grad
        # about ten roundings to bf16 (2^-9 each, root mean square) on the way from x to a gradient
        assert float((got - want).norm() / want.norm()) < 10 * 2 ** -9, n


def test_ragged_attention_has_gradients(layer_mod):
    import torch

    from paper_2609_29219_gb300 import autograd
    lens = [30, 50]
    mk = lambda h: torch.randn((80, h, 64), device="cuda").bfloat16().requires_grad_()  # noqa: E731
    q, k, v = mk(4), mk(2), mk(2)
    cu = torch.tensor([0, 30, 80], dtype=torch.int32, device="cuda")
    o, lse = autograd.attention_varlen(q, k, v, cu, cu, 50, 50, causal=True)
    (o.float().sum() + lse.sum()).backward()
    for i, (a, e) in enumerate(((0, 30), (30, 80))):
        part = [t.detach()[a:e].transpose(0, 1).unsqueeze(0).contiguous().requires_grad_() for t in (q, k, v)]
        oo, ll = autograd.attention(*part, causal=True)
        (oo.float().sum() + ll.sum()).backward()
        for t, p in zip((q, k, v), part):
            # the same kernels on the same rows, other tiles: two roundings apart at most
            diff = (t.grad[a:e].float() - p.grad[0].transpose(0, 1).float()).abs()
            assert float(diff.max()) <= 2 ** -6 * float(p.grad.float().abs().max()), (i, lens)
