"""Sizes and factors that are numbers of numpy's or torch's: taken by the training and serving entry
points as the older ones take them, from either way in."""
import pytest

from tests.test_gpu_given_stream import loom  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way", ["compiled", "python"])
@pytest.mark.parametrize("integer", ["int64", "tensor"])
def test_numbers_of_other_types(loom, monkeypatch, integer, way):  # noqa: F811
    import numpy as np
    import torch
    if way == "python":
        monkeypatch.setattr(loom, "_fast", None)
    i = np.int64 if integer == "int64" else torch.tensor
    f = np.float32 if integer == "int64" else torch.tensor
    gen = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    fq, fk, fdo = mk(24, 2, 64), mk(24, 1, 64), mk(24, 2, 64)
    cu = torch.tensor([0, 24], dtype=torch.int32, device="cuda")
    fo, fl = loom.loom_attn_fwd_varlen(fq, fk, fk, cu, cu, i(24), scale=f(0.25), return_lse=True)
    q, k, do = (t.view(1, -1, 24, 64) for t in (fq, fk, fdo))
    o, lse = loom.loom_attn_fwd(q, k, k, scale=f(0.25), return_lse=True)
    w, t, pos = mk(64), torch.rand((24, 32), device="cuda"), torch.arange(24, dtype=torch.int32, device="cuda")
    norm = (mk(24, 256), w, w, t, t)

    def cached(heads, eps):
        c = torch.zeros((2, 2, 16, 1, 64), dtype=torch.bfloat16, device="cuda")
        return loom.loom_qkv_norm_rope_cache(*norm, pos, pos, c[0], c[1], heads, eps=eps), c

    pairs = [
        (lambda s: loom.loom_attn_bwd(do, q, k, k, o, lse, scale=s), (0.25,), (f(0.25),)),
        (lambda a, b, s: loom.loom_attn_bwd_varlen(fdo, fq, fk, fk, fo, fl, cu, cu, a, b, scale=s), (24, 24, 0.25),
         (i(24), i(24), f(0.25))),
        (lambda h, g, s, e: loom.loom_qkv_norm_rope(*norm, h, g, seq_len=s, eps=e), (2, 1, 8, 0.5), (i(2), i(1), i(8), f(0.5))),
        (cached, (2, 0.5), (i(2), f(0.5))),
        (lambda e: loom.loom_qkv_norm_rope_bwd(fdo, fk, fk, *norm, pos, eps=e), (0.5,), (f(0.5),)),
    ]
    for call, plain, other in pairs:
        for a, b in zip(call(*plain), call(*other)):
            assert a.shape == b.shape and torch.equal(a, b)
