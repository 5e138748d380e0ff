"""Flags whose truth value raises: the exception is the caller's, from either way in."""
import pytest

from tests.test_gpu_given_stream import loom  # noqa: F401

pytestmark = pytest.mark.gpu


class Broken:
    def __bool__(self):
        raise KeyError("no truth value")


@pytest.mark.parametrize("way", ["compiled", "python"])
def test_a_flag_that_raises(loom, monkeypatch, way):  # noqa: F811
    import torch
    if way == "python":
        monkeypatch.setattr(loom, "_fast", None)
    z = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    w, t, pos = z(64), torch.zeros((8, 32), device="cuda"), torch.arange(8, dtype=torch.int32, device="cuda")
    q, k, lse, cu = z(1, 2, 8, 64), z(1, 1, 8, 64), torch.zeros((1, 2, 8), device="cuda"), pos[[0, 7]].contiguous()
    norm = (z(8, 256), w, w, t, t)
    calls = [lambda: loom.loom_qkv_norm_rope(*norm, 2, 1, pos, interleaved=Broken()),
             lambda: loom.loom_qkv_norm_rope_cache(*norm, pos, pos, z(1, 8, 1, 64), z(1, 8, 1, 64), 2, interleaved=Broken()),
             lambda: loom.loom_qkv_norm_rope_bwd(z(8, 2, 64), z(8, 1, 64), z(8, 1, 64), *norm, pos, interleaved=Broken()),
             lambda: loom.loom_attn_bwd(q, q, k, k, q, lse, causal=Broken()),
             lambda: loom.loom_attn_bwd_varlen(z(7, 2, 64), z(7, 2, 64), z(7, 1, 64), z(7, 1, 64), z(7, 2, 64),
                                               torch.zeros((2, 7), device="cuda"), cu, cu, 7, 7, causal=Broken())]
    for f in calls:
        with pytest.raises(KeyError, match="no truth value"):
            f()
    torch.cuda.synchronize()


@pytest.mark.parametrize("way", ["compiled", "python"])
def test_gradients_that_are_no_tensors_are_named(loom, monkeypatch, way):  # noqa: F811
    import torch
    if way == "python":
        monkeypatch.setattr(loom, "_fast", None)
    z = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    w, t = z(64), torch.zeros((8, 32), device="cuda")
    grads = {"dq": z(8, 2, 64), "dk": z(8, 1, 64), "dv": z(8, 1, 64)}
    for name in grads:
        for bad in (None, [1.0]):
            with pytest.raises(TypeError, match=name):
                loom.loom_qkv_norm_rope_bwd(*{**grads, name: bad}.values(), z(8, 256), w, w, t, t)
