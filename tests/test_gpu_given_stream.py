"""Calls on a stream given: what they allocate belongs to that stream, not to the current one."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loom():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_29219_gb300 as m
    m._torch()
    return m


def _calls(loom):
    """name -> (call(stream), its input tensors)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(2)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, v, do = mk(1, 8, 700, 64), mk(1, 1, 900, 64), mk(1, 1, 900, 64), mk(1, 8, 700, 64)
    o, lse = loom.loom_attn_fwd(q, k, v, return_lse=True)
    flat = lambda t: t[0].transpose(0, 1).contiguous()  # noqa: E731
    fq, fk, fv, fdo, fo, fl = flat(q), flat(k), flat(v), flat(do), flat(o), lse[0].contiguous()
    cq, ck = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 700], [0, 900]))
    q1, kc, vc = mk(2, 8, 1, 64), mk(2, 2, 2048, 64), mk(2, 2, 2048, 64)
    table = torch.arange(2 * 32, dtype=torch.int32, device="cuda").view(2, 32)
    lens = torch.tensor([2048, 2048], dtype=torch.int32, device="cuda")
    kp, vp = (t.view(2, 2, 32, 64, 64).transpose(1, 2).reshape(64, 2, 64, 64) for t in (kc, vc))
    rows, w, cos, sin = mk(40, 8 * 64), mk(64), torch.rand((50, 16), device="cuda"), torch.rand((50, 16), device="cuda")
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    norm = (rows, w, w, cos, sin)
    c1, c2 = (torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gq, gk, gv = mk(40, 4, 64), mk(40, 2, 64), mk(40, 2, 64)
    a, b = mk(64, 128), mk(128, 192)
    return {
        "fwd": (lambda s: loom.loom_attn_fwd(q, k, v, return_lse=True, stream=s), (q, k, v)),
        "varlen": (lambda s: loom.loom_attn_fwd_varlen(fq, fk, fv, cq, ck, 700, return_lse=True, stream=s), (fq, fk, fv, cq, ck)),
        "decode": (lambda s: loom.loom_attn_decode(q1, kc, vc, lens, num_splits=4, return_lse=True, stream=s), (q1, kc, vc, lens)),
        "noalloc": (lambda s: loom.loom_attn_decode_noalloc(q1, kc, vc, lens, return_lse=True, stream=s), (q1, kc, vc, lens)),
        "paged": (lambda s: loom.loom_attn_decode_paged(q1, kp, vp, table, lens, num_splits=4, return_lse=True, stream=s,
                                                        layout="hnd"), (q1, kp, vp, table, lens)),
        "gemm": (lambda s: loom.loom_gemm_bf16(a, b, stream=s), (a, b)),
        "bwd": (lambda s: loom.loom_attn_bwd(do, q, k, v, o, lse, dlse=lse, stream=s), (do, q, k, v, o, lse)),
        "bwd_varlen": (lambda s: loom.loom_attn_bwd_varlen(fdo, fq, fk, fv, fo, fl, cq, ck, 700, 900, stream=s),
                       (fdo, fq, fk, fv, fo, fl, cq, ck)),
        "norm": (lambda s: loom.loom_qkv_norm_rope(*norm, 4, 2, pos, stream=s), (*norm, pos)),
        "cache": (lambda s: loom.loom_qkv_norm_rope_cache(*norm, pos, pos, c1, c2, 4, layout="hnd", stream=s),
                  (*norm, pos, c1, c2)),
        "norm_bwd": (lambda s: loom.loom_qkv_norm_rope_bwd(gq, gk, gv, *norm, pos, stream=s), (gq, gk, gv, *norm, pos)),
    }


NAMES = ("fwd", "varlen", "decode", "noalloc", "paged", "gemm", "bwd", "bwd_varlen", "norm", "cache", "norm_bwd")


class NoLaunch:
    """The library, except that its entry points keep their arguments and do nothing."""

    def __init__(self, lib):
        self.lib, self.args = lib, None

    def __getattr__(self, name):
        f = getattr(self.lib, name)
        if name.endswith("_bytes") or name.startswith("loom_debug"):
            return f

        def entry(*args):
            self.args = args
            return 0
        return entry


def _owner(pointer):
    """The stream that the allocator keeps a pointer's memory for (None: it is not the allocator's)."""
    import torch
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= pointer < s["address"] + s["total_size"]:
            return s["stream"]
    return None


def _tensors(out):
    return list(out) if isinstance(out, tuple) else [out]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_and_scratch_are_the_streams_own(loom, monkeypatch, name):
    """Without a launch: the owners of every pointer that the call hands over and did not get."""
    import torch
    call, inputs = _calls(loom)[name]
    side = torch.cuda.Stream()
    lib = NoLaunch(loom.capi())
    monkeypatch.setattr(loom, "_lib", lib)
    for given in (side, side.cuda_stream):
        out = call(given)
        had = {t.data_ptr() for t in inputs} | {side.cuda_stream}
        made = [a for a in lib.args if isinstance(a, int) and a > 1 << 24 and a not in had and _owner(a) is not None]
        assert len(made) >= len(_tensors(out)) - (name == "cache")
        assert {_owner(a) for a in made} == {side.cuda_stream}
        assert {t.data_ptr() for t in _tensors(out)} <= set(made)


@pytest.mark.parametrize("name", NAMES)
def test_what_the_current_stream_allocates_meanwhile_does_not_matter(loom, name):
    """The stream is busy; the current one takes and fills memory of the sizes of the call's scratch."""
    import torch
    call, _ = _calls(loom)[name]
    want = [t.clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for given in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        out = call(given)
        assert not side.query()
        hold = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in [1 << i for i in range(9, 25)] * 4]
        torch.cuda.current_stream().synchronize()
        side.synchronize()
        del hold
        assert all(torch.equal(a, b) for a, b in zip(want, _tensors(out)))
    loom.loom_attn_check_error()


@pytest.mark.parametrize("name", ["decode", "bwd", "norm"])
def test_the_default_streams_handle(loom, name):
    import torch
    call, _ = _calls(loom)[name]
    want = [t.clone() for t in _tensors(call(None))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = call(0)
        assert all(_owner(t.data_ptr()) == 0 for t in _tensors(got))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, _tensors(got)))
