"""The compiled binding of the training and serving entry points against the package's Python code,
and where a program watches torch's allocations."""
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
    """Calls of each entry point, with and without the optional arguments."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    mk = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    q, k, v, do = mk(2, 4, 70, 64), mk(2, 2, 90, 64), mk(2, 2, 90, 64), mk(2, 4, 70, 64)
    o, lse = loom.loom_attn_fwd(q, k, v, causal=True, return_lse=True)
    flat = lambda t: t.transpose(1, 2).reshape(-1, t.shape[1], 64).contiguous()  # noqa: E731
    cq = torch.tensor([0, 70, 140], dtype=torch.int32, device="cuda")
    ck = torch.tensor([0, 90, 180], dtype=torch.int32, device="cuda")
    lf = lse.transpose(0, 1).reshape(4, 140).contiguous()
    rows = mk(12, 8 * 64 + 8)
    qw, kw = torch.nn.Parameter(mk(64)), mk(64)
    cos, sin = torch.rand((50, 16), device="cuda"), torch.rand((50, 16), device="cuda")
    pos = torch.arange(12, dtype=torch.int32, device="cuda")
    norm = (rows[:, :512], qw, kw, cos, sin)

    def cached():
        caches = torch.zeros((2, 3, 2, 4, 64), dtype=torch.bfloat16, device="cuda")
        return loom.loom_qkv_norm_rope_cache(*norm, pos, pos, caches[0], caches[1], 4, layout="hnd"), caches

    return [lambda: loom.loom_attn_bwd(do, q, k, v, o, lse, causal=True),
            lambda: loom.loom_attn_bwd(do, q, k, v, o, lse, dlse=lse, scale=0.3),
            lambda: loom.loom_attn_bwd_varlen(*map(flat, (do, q, k, v, o)), lf, cq, ck, 70, 90, causal=True, dlse=lf),
            lambda: loom.loom_qkv_norm_rope(*norm, 4, 2, pos, interleaved=True),
            lambda: loom.loom_qkv_norm_rope(*norm, 4, 2, seq_len=6, eps=1e-3), cached,
            lambda: loom.loom_qkv_norm_rope_bwd(mk(12, 4, 64).zero_().add_(1), kv := mk(12, 2, 64).zero_().add_(2), kv, *norm, pos),
            lambda: loom.loom_qkv_norm_rope_bwd(mk(2, 4, 6, 64).zero_().add_(1), kv := mk(2, 2, 6, 64).zero_().add_(2), kv, *norm)]


def test_both_ways_give_the_same(loom, monkeypatch):
    import torch
    if loom._fast is None:
        pytest.skip("the compiled binding was not built")
    calls = _calls(loom)
    compiled = [f() for f in calls]
    monkeypatch.setattr(loom, "_fast", None)
    for f, a in zip(calls, compiled):
        for x, y in zip(a, f()):
            assert x.shape == y.shape and x.stride() == y.stride() and x.dtype == y.dtype and torch.equal(x, y)
    loom.loom_attn_check_error()


def test_the_compiled_binding_takes_the_common_case(loom, monkeypatch):
    """Every call above goes the short way (the Python code's checks are not reached)."""
    if loom._fast is None:
        pytest.skip("the compiled binding was not built")
    calls = _calls(loom)
    for n in ("_bwd_fine", "_norm_operands"):
        monkeypatch.setattr(loom, n, lambda *a, n=n: pytest.fail(f"{n} was reached"))
    for f in calls:
        f()


def test_a_dispatch_mode_sees_the_outputs(loom):
    import torch
    from torch.utils._python_dispatch import TorchDispatchMode
    seen = []

    class Watch(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            seen.append(str(func))
            return func(*args, **(kwargs or {}))

    f = _calls(loom)[0]
    with Watch():
        f()
    assert sum("empty" in s for s in seen) >= 4  # three gradients and the workspace


def test_current_stream_is_taken(loom):
    import torch
    f = _calls(loom)[0]
    want = f()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        got = f()
        assert not side.query()  # queued behind the sleep
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_errors_are_the_same(loom, monkeypatch):
    import torch
    z = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    lse = torch.zeros((1, 2, 4), device="cuda")
    bad = [lambda: loom.loom_attn_bwd(z(1, 2, 4, 32), z(1, 2, 4, 32), z(1, 2, 4, 32), z(1, 2, 4, 32), z(1, 2, 4, 32), lse),
           lambda: loom.loom_attn_bwd(z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), lse, scale=-1.0),
           lambda: loom.loom_attn_bwd(z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 3, 64), z(1, 2, 3, 64), z(1, 2, 4, 64), lse, causal=True),
           lambda: loom.loom_attn_bwd(z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), None, lse),
           lambda: loom.loom_attn_bwd(z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 4, 64), z(1, 2, 5, 64), z(1, 2, 4, 64), lse),
           lambda: loom.loom_qkv_norm_rope(z(3, 512), z(64), z(64), lse[0], lse[0], 4, 2)]
    for way in ("compiled", "python"):
        if way == "python":
            monkeypatch.setattr(loom, "_fast", None)
        kinds = []
        for f in bad:
            with pytest.raises(Exception) as e:
                f()
            kinds.append((type(e.value), str(e.value)))
        if way == "compiled":
            first = kinds
    assert first == kinds


def test_out_of_memory_is_torchs_error(loom, monkeypatch):
    """Where an output cannot be allocated both ways raise what torch raises, and the next call works."""
    import torch
    x = torch.randn((4096, 8 * 128), device="cuda").bfloat16()
    w, cos = torch.ones(128, device="cuda").bfloat16(), torch.rand((4096, 32), device="cuda")
    call = lambda: loom.loom_qkv_norm_rope(x, w, w, cos, cos, 4, 2)  # noqa: E731
    want = [t.clone() for t in call()]
    for way in ("compiled", "python"):
        if way == "python":
            monkeypatch.setattr(loom, "_fast", None)
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.set_per_process_memory_fraction(1e-6)
        try:
            with pytest.raises(torch.OutOfMemoryError):
                hold = [call() for _ in range(64)]  # noqa: F841
        finally:
            torch.cuda.set_per_process_memory_fraction(1.0)
        assert all(torch.equal(a, b) for a, b in zip(want, call()))


def test_a_function_transform_is_refused_both_ways(loom, monkeypatch):
    """A batched tensor of torch.func has no memory of its own: the call names that, it reads nothing."""
    import torch
    w, cos = torch.ones(64, device="cuda").bfloat16(), torch.rand((8, 32), device="cuda")
    x = torch.randn((3, 8, 4 * 64), device="cuda").bfloat16()
    for way in ("compiled", "python"):
        if way == "python":
            monkeypatch.setattr(loom, "_fast", None)
        with pytest.raises(Exception):
            torch.func.vmap(lambda t: loom.loom_qkv_norm_rope(t, w, w, cos, cos, 2, 1)[0])(x)
