"""Tensors of a call on more than one device, or not on the current one: refused by name, before
anything is launched.  (One GPU is enough: the package is told of another, and a tensor says that
it is there.)"""
import pytest

from tests.test_gpu_given_stream import NAMES, NoLaunch, loom  # noqa: F401

pytestmark = pytest.mark.gpu


def _elsewhere(t):
    import torch

    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1

        @property
        def device(self):
            return torch.device("cuda", 1)
    return t.as_subclass(Elsewhere)


def _calls(loom):  # noqa: F811
    """name -> (function, its tensors by name, the rest)."""
    import torch
    mk = lambda *s: torch.ones(s, device="cuda").bfloat16()  # noqa: E731
    f32 = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    u8 = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    q, k, one, cache = mk(2, 4, 64, 64), mk(2, 2, 64, 64), mk(2, 4, 1, 64), mk(2, 2, 128, 64)
    fq, fk = mk(64, 4, 64), mk(64, 2, 64)
    norm = {"qkv": mk(8, 512), "q_weight": mk(64), "k_weight": mk(64), "cos": f32(8, 16), "sin": f32(8, 16)}
    pos = {"positions": i32(*range(8))}
    bwd = lambda q, k, lse: {"do": q, "q": q.clone(), "k": k, "v": k.clone(), "o": q.clone(), "lse": lse, "dlse": lse.clone(),  # noqa: E731
                             "dq": q.clone(), "dk": k.clone(), "dv": k.clone(), "workspace": u8}
    heads = {"num_heads": 4, "num_kv_heads": 2}
    cu = {"cu_seqlens_q": i32(0, 64), "cu_seqlens_k": i32(0, 64)}
    return {
        "fwd": (loom.loom_attn_fwd, {"q": q, "k": k, "v": k.clone(), "o": q.clone(), "lse": f32(2, 4, 64)}, {}),
        "varlen": (loom.loom_attn_fwd_varlen, {"q": fq, "k": fk, "v": fk.clone(), **cu, "o": fq.clone(), "lse": f32(4, 64)},
                   {"max_seqlen_q": 64}),
        "decode": (loom.loom_attn_decode, {"q": one, "k_cache": cache, "v_cache": cache.clone(), "seqlens_k": i32(128, 128),
                                           "o": one.clone(), "lse": f32(2, 4), "workspace": u8}, {}),
        "noalloc": (loom.loom_attn_decode_noalloc, {"q": one, "k_cache": cache, "v_cache": cache.clone(),
                                                    "seqlens_k": i32(128, 128), "o": one.clone(), "lse": f32(2, 4)}, {}),
        "paged": (loom.loom_attn_decode_paged, {"q": one, "k_cache": cache.view(2, 2, 128, 64), "v_cache": cache.clone(),
                                                "block_table": i32([0], [1]), "seqlens_k": i32(128, 128), "o": one.clone(),
                                                "lse": f32(2, 4), "workspace": u8}, {"layout": "hnd"}),
        "gemm": (loom.loom_gemm_bf16, {"a": mk(16, 64), "b": mk(64, 32), "c": mk(16, 32)}, {}),
        "bwd": (loom.loom_attn_bwd, bwd(q, k, f32(2, 4, 64)), {}),
        "bwd_varlen": (loom.loom_attn_bwd_varlen, {**bwd(fq, fk, f32(4, 64)), **cu}, {"max_seqlen_q": 64, "max_seqlen_k": 64}),
        "norm": (loom.loom_qkv_norm_rope, {**norm, **pos, "q": mk(8, 4, 64), "k": mk(8, 2, 64), "v": mk(8, 2, 64)}, heads),
        "cache": (loom.loom_qkv_norm_rope_cache, {**norm, **pos, "slots": i32(*range(8)), "k_cache": cache,
                                                  "v_cache": cache.clone(), "q": mk(8, 4, 64)}, {"num_heads": 4, "layout": "hnd"}),
        "norm_bwd": (loom.loom_qkv_norm_rope_bwd, {"dq": mk(8, 4, 64), "dk": mk(8, 2, 64), "dv": mk(8, 2, 64), **norm, **pos,
                                                   "dqkv": mk(8, 512), "dq_weight": f32(64), "dk_weight": f32(64),
                                                   "workspace": u8}, {}),
    }


@pytest.mark.parametrize("name", NAMES)
def test_a_tensor_elsewhere_is_named(loom, monkeypatch, name):  # noqa: F811
    f, tensors, rest = _calls(loom)[name]
    lib = NoLaunch(loom.capi())
    monkeypatch.setattr(loom, "_lib", lib)
    monkeypatch.setattr(loom, "_several", True, raising=False)
    f(**tensors, **rest)
    for one in tensors:
        lib.args = None
        with pytest.raises(ValueError, match="cuda:1"):
            f(**{n: _elsewhere(t) if n == one else t for n, t in tensors.items()}, **rest)
        assert lib.args is None, one


@pytest.mark.parametrize("name", NAMES)
def test_the_current_device_must_be_the_tensors(loom, monkeypatch, name):  # noqa: F811
    f, tensors, rest = _calls(loom)[name]
    lib = NoLaunch(loom.capi())
    monkeypatch.setattr(loom, "_lib", lib)
    monkeypatch.setattr(loom, "_several", True, raising=False)
    monkeypatch.setattr(loom, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="current device"):
        f(**tensors, **rest)
    assert lib.args is None
