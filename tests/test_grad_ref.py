"""The 64-bit formulas of tests/grad_ref.py against central differences (CPU)."""
import pytest
import torch

from tests import grad_ref as ref


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float64)


@pytest.mark.parametrize("causal,sq,skv", [(False, 5, 7), (True, 4, 9), (True, 7, 3)])
@pytest.mark.parametrize("with_dlse", [False, True])
def test_attention_gradients_against_differences(causal, sq, skv, with_dlse):
    gen = torch.Generator().manual_seed(1)
    q, k, v = _rand(gen, 4, sq, 8), _rand(gen, 2, skv, 8), _rand(gen, 2, skv, 8)
    do, dl = _rand(gen, 4, sq, 8), _rand(gen, 4, sq)

    def loss(q, k, v):
        o, lse = ref.attention(q, k, v, causal, 0.3)
        fin = torch.isfinite(lse)
        return (do * o).sum() + ((dl * torch.where(fin, lse, 0.0)).sum() if with_dlse else 0.0)

    o, lse = ref.attention(q, k, v, causal, 0.3)
    grads, _ = ref.attention_grads(do, q, k, v, o, lse, dl if with_dlse else None, causal, 0.3)
    h = 1e-5
    for i, x in enumerate((q, k, v)):
        u = _rand(gen, *x.shape)
        at = lambda e: loss(*[y + e * u if j == i else y for j, y in enumerate((q, k, v))])  # noqa: E731
        # truncation about h^2 times a third derivative of order 10, rounding 1e-15 / h
        assert abs((at(h) - at(-h)) / (2 * h) - (grads[i] * u).sum()) < 1e-8


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [4, 8])
def test_norm_rope_gradients_against_differences(interleaved, R):
    gen = torch.Generator().manual_seed(2)
    x, w, dy = _rand(gen, 3, 2, 8), _rand(gen, 8), _rand(gen, 3, 2, 8)
    angle = _rand(gen, 3, R // 2)
    c, s = angle.cos(), angle.sin()
    (dx, dw), _ = ref.norm_rope_grads(dy, x, w, c, s, R, interleaved, 1e-6)
    loss = lambda x, w: (dy * ref.norm_rope(x, w, c, s, R, interleaved, 1e-6)).sum()  # noqa: E731
    h = 1e-5
    u, uw = _rand(gen, *x.shape), _rand(gen, 8)
    assert abs((loss(x + h * u, w) - loss(x - h * u, w)) / (2 * h) - (dx * u).sum()) < 1e-8
    assert abs((loss(x, w + h * uw) - loss(x, w - h * uw)) / (2 * h) - (dw * uw).sum()) < 1e-8
