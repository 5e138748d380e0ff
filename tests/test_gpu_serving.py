"""The serving calls together -- a step's plan, norm and rotation into the cache, attention over it -- and what
they share with the other Python calls: compiled and plain bindings, streams, devices, failed waits."""
import pytest

from tests import chunk_ref as ref
from tests.test_gpu_chunk import Case, _check
from tests.test_gpu_devices import _elsewhere
from tests.test_gpu_given_stream import NoLaunch, _owner, _tensors, loom  # noqa: F401

pytestmark = pytest.mark.gpu


def _ints(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_layer_served_in_chunks_matches_its_prefill(loom):  # noqa: F811
    """Requests of unlike lengths, in chunks of unlike sizes, one of them ended and begun anew in between."""
    import torch
    from paper_2609_29219_gb300 import layer as mod
    layer = mod.AttentionLayer(model=256, Hq=8, Hkv=2, D=64, positions=256, seed=0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    texts = [torch.randn((n, 256), generator=gen, device="cuda").bfloat16() for n in (150, 33, 90, 200)]
    with torch.no_grad():
        want = [layer.forward(torch.cat((x, x.new_zeros(-len(x) % 8, 256)))[None])[0, :len(x)].float() for x in texts]
    cache = mod.RequestCache(3, 40, 256, 2, 64)
    at, row_of, got = [0] * 4, [0, 1, 2], [[] for _ in texts]
    steps = [(100, 1, 0), (1, 32, 7), (49, -1, 1), (0, 120, 82), (0, 80, 0)]  # row 1's second text begins in the fourth
    for new in steps:
        rows = []
        for r, n in enumerate(new):
            if n < 0:
                row_of[r] = 3
            elif n:
                t = row_of[r]
                rows.append((t, texts[t][at[t]:at[t] + n]))
                at[t] += n
        x = torch.cat([x for _, x in rows] + [texts[0].new_zeros(5, 256)])  # five rows of padding
        y = layer.serve(x, cache, _ints(*new))
        for (t, part), out in zip(rows, y[:-5].split([len(p) for _, p in rows])):
            got[t].append(out.float())
    loom.loom_attn_check_error()
    assert at == [150, 33, 90, 200]
    for w, g in zip(want, got):
        # both round q, k, v, P, O and the result to bf16: a few units of 2^-8 of the largest value
        assert float((torch.cat(g) - w).abs().max()) <= 2 ** -5 * float(w.abs().max())
    held = sum(ref.pages(n, 16) for n in cache.lens.tolist())
    assert cache.lens.tolist() == [150, 200, 90] and int(cache.free_count) == 40 - held


def test_a_step_with_positions_on_several_axes(loom):  # noqa: F811
    """The plan's slots, the rotated keys in them, and the attention of what the cache then holds, in 64 bits."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    Hq, Hkv, D, T, page, pages = 14, 2, 128, 150, 16, 40
    k, v = (torch.full((pages, page, Hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, lens = torch.full((3, 20), -1, dtype=torch.int32, device="cuda"), _ints(0, 0, 0)
    free, count = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32), _ints(pages)
    w, cos, sin = torch.rand(D, generator=gen, device="cuda") + 0.5, *torch.randn((2, 300, D // 2), generator=gen, device="cuda")
    axis = tuple(i % 3 for i in range(D // 2))
    for new in ([100, 1, 40], [1, 130, 9], [20, 1, 0]):
        qkv = torch.randn((T, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").bfloat16()
        cu, _, pos, slots, granted = loom.loom_paged_plan(_ints(*new), lens, table, free, count, T, page, seqlens_k=lens)
        assert granted.tolist() == new and len(set(slots[:sum(new)].tolist())) == sum(new)
        where = torch.stack((pos, pos // 7, pos % 7))
        q = loom.loom_qkv_norm_rope_cache(qkv, w, w, cos, sin, where, slots, k, v, Hq, pair_axis=axis)
        fresh = loom.loom_qkv_norm_rope(qkv, w, w, cos, sin, Hq, Hkv, where, pair_axis=axis)
        n = sum(new)
        assert torch.equal(q, fresh[0])
        for cache, x in ((k, fresh[1]), (v, fresh[2])):
            assert torch.equal(cache.view(-1, Hkv, D)[slots[:n].long()], x[:n])
        o, lse = loom.loom_attn_chunk_paged(q, k, v, table, cu, lens, return_lse=True)
        _check(o, lse, ref.chunk(q.cpu(), k.cpu(), v.cpu(), table.cpu(), cu.tolist(), lens.tolist(), True, D ** -0.5, "nhd"), str(new))


def test_a_whole_step_captured_and_replayed(loom):  # noqa: F811
    """One graph plans, rotates, attends and runs again on what it left: a prompt, then token after token."""
    import torch
    from paper_2609_29219_gb300 import layer as mod
    layer = mod.AttentionLayer(model=128, Hq=4, Hkv=2, D=64, positions=128, seed=2)
    xs = torch.randn((6, 40, 128), device="cuda").bfloat16()
    news = [[30, 0], [1, 38], [1, 1], [0, 1], [8, -1], [0, 40]]
    caches = [mod.RequestCache(2, 12, 96, 2, 64) for _ in range(2)]
    x, new = torch.zeros((40, 128), dtype=torch.bfloat16, device="cuda"), _ints(0, 0)
    layer.serve(x, caches[0], new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = layer.serve(x, caches[0], new)
    for data, n in zip(xs, news):
        x.copy_(data)
        new.copy_(_ints(*n))
        graph.replay()
        want = layer.serve(data, caches[1], _ints(*n))
        real = sum(max(a, 0) for a in n)
        assert torch.equal(y[:real], want[:real])
        for name in ("lens", "table", "free_count"):
            assert torch.equal(getattr(caches[0], name), getattr(caches[1], name)), name


@pytest.mark.parametrize("ql,kl", [([1], [3000]), ([300], [2000]), ([1, 1, 200], [4000, 4000, 300])])
@pytest.mark.parametrize("D", [64, 128])
def test_a_wait_that_gives_up(loom, ql, kl, D):  # noqa: F811
    """A tile that is never loaded: the call reports it, and the next one on the same workspace is right."""
    import torch
    c = Case(ql, kl, 16, 2, D)
    d, n = c.device(), loom.loom_attn_chunk_paged_workspace_bytes(len(ql), 16, 2, sum(ql), D)
    ws = torch.full((n,), 7, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        loom.loom_debug_set_timeout_ns(50_000_000)
        loom.loom_debug_inject(5)
        try:
            loom.loom_attn_chunk_paged(*d, workspace=ws)
            with pytest.raises(loom.LoomError, match="TIMEOUT"):
                loom.loom_attn_check_error()
        finally:
            loom.loom_debug_inject(0)
            loom.loom_debug_set_timeout_ns(0)
        for _ in range(2):
            o, lse = loom.loom_attn_chunk_paged(*d, workspace=ws, return_lse=True)
            loom.loom_attn_check_error()
            _check(o, lse, c.exact(True))


# ------------------------------------------------------------------ the Python calls
def _calls(loom):  # noqa: F811
    """name -> (function, its tensors by name, the rest, outputs that it may be given)."""
    import torch
    mk = lambda *s: torch.randn(s, device="cuda").bfloat16()  # noqa: E731
    c = Case([30, 1], [300, 2000], 8, 2, 64)
    q, k, v, table, cu, lens = c.device()
    plan = {"new_lens": _ints(3, -1, 20), "lens": _ints(15, 40, 0), "block_table": _ints(0, 9, 9, 1, 2, 3, 9, 9, 9).view(3, 3),
            "free_pages": torch.arange(4, 12, dtype=torch.int32, device="cuda"), "free_count": _ints(5)}
    norm = {"qkv": mk(12, 8 * 64), "q_weight": mk(64), "k_weight": mk(64), "cos": torch.rand((20, 16), device="cuda"),
            "sin": torch.rand((20, 16), device="cuda"), "positions": torch.randint(0, 20, (3, 12), device="cuda", dtype=torch.int32)}
    axis = tuple(i % 3 for i in range(16))
    caches = [mk(2, 2, 16, 64) for _ in range(2)]
    slots = torch.randperm(32, device="cuda")[:12].to(torch.int32)
    return {
        "chunk": (loom.loom_attn_chunk_paged, {"q": q, "k_cache": k, "v_cache": v, "block_table": table, "cu_seqlens_q": cu,
                                               "seqlens_k": lens}, {"return_lse": True},
                  {"o": q.clone(), "lse": torch.zeros((8, 31), device="cuda"), "workspace": torch.zeros(41 << 20, dtype=torch.uint8, device="cuda")}),
        "plan": (loom.loom_paged_plan, plan, {"num_tokens": 25, "page_size": 16},
                 {"free_count_out": _ints(0), "seqlens_k": _ints(0, 0, 0), "cu_seqlens": _ints(0, 0, 0, 0),
                  "positions": _ints(*[0] * 25), "slots": _ints(*[0] * 25), "granted": _ints(0, 0, 0)}),
        "axes": (loom.loom_qkv_norm_rope, norm, {"num_heads": 4, "num_kv_heads": 2, "pair_axis": axis},
                 {"q": mk(12, 4, 64), "k": mk(12, 2, 64), "v": mk(12, 2, 64)}),
        "axes_cache": (loom.loom_qkv_norm_rope_cache, {**norm, "slots": slots, "k_cache": caches[0], "v_cache": caches[1]},
                       {"num_heads": 4, "pair_axis": axis, "layout": "hnd"}, {"q": mk(12, 4, 64)}),
        "axes_bwd": (loom.loom_qkv_norm_rope_bwd, {"dq": mk(12, 4, 64), "dk": mk(12, 2, 64), "dv": mk(12, 2, 64), **norm},
                     {"pair_axis": axis}, {"dqkv": mk(12, 8 * 64), "dq_weight": torch.zeros(64, device="cuda"),
                                           "dk_weight": torch.zeros(64, device="cuda"),
                                           "workspace": torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")}),
    }


NAMES = ("chunk", "plan", "axes", "axes_cache", "axes_bwd")


def _run(f, tensors, rest, outs=None):
    """The call on copies of what it updates: its results and those."""
    import torch
    t = {n: x.clone() for n, x in tensors.items()}
    r = _tensors(f(**t, **rest, **{n: x.clone() for n, x in (outs or {}).items()}))
    torch.cuda.synchronize()
    return r + [t[n] for n in ("block_table", "k_cache", "v_cache") if n in t]


@pytest.mark.parametrize("name", NAMES)
def test_all_ways_give_the_same(loom, monkeypatch, name):  # noqa: F811
    """Compiled binding, Python code, outputs given, a stream given; and axes as a list or tensor."""
    import torch
    f, tensors, rest, outs = _calls(loom)[name]
    want = _run(f, tensors, rest)
    ways = [lambda: _run(f, tensors, rest, outs), lambda: _run(f, tensors, {**rest, "stream": torch.cuda.current_stream()})]
    if "pair_axis" in rest:
        ways += [lambda: _run(f, tensors, {**rest, "pair_axis": list(rest["pair_axis"])}),
                 lambda: _run(f, tensors, {**rest, "pair_axis": torch.tensor(rest["pair_axis"])})]

    def plain():
        monkeypatch.setattr(loom, "_fast", None)
        return _run(f, tensors, rest)
    for way in (*ways, plain):
        for a, b in zip(want, way()):
            assert a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    loom.loom_attn_check_error()


@pytest.mark.parametrize("name", NAMES)
def test_the_compiled_binding_takes_the_common_case(loom, monkeypatch, name):  # noqa: F811
    if loom._fast is None:
        pytest.skip("the compiled binding was not built")
    f, tensors, rest, _ = _calls(loom)[name]
    for n in ("_ptr", "_dev_ptr", "_norm_operands"):
        monkeypatch.setattr(loom, n, lambda *a, n=n: pytest.fail(f"{n} was reached"))
    f(**tensors, **rest)


@pytest.mark.parametrize("name", NAMES)
def test_outputs_and_scratch_are_the_given_streams_own(loom, monkeypatch, name):  # noqa: F811
    import torch
    f, tensors, rest, _ = _calls(loom)[name]
    side = torch.cuda.Stream()
    lib = NoLaunch(loom.capi())
    monkeypatch.setattr(loom, "_lib", lib)
    for given in (side, side.cuda_stream):
        out = f(**tensors, **rest, stream=given)
        had = {t.data_ptr() for t in tensors.values()} | {side.cuda_stream}
        made = [a for a in lib.args if isinstance(a, int) and a > 1 << 24 and a not in had and _owner(a) is not None]
        assert {_owner(a) for a in made} == {side.cuda_stream}
        assert {t.data_ptr() for t in _tensors(out)} <= set(made)


@pytest.mark.parametrize("name", NAMES)
def test_a_tensor_elsewhere_is_named(loom, monkeypatch, name):  # noqa: F811
    f, tensors, rest, outs = _calls(loom)[name]
    tensors = {**tensors, **outs}
    lib = NoLaunch(loom.capi())
    monkeypatch.setattr(loom, "_lib", lib)
    monkeypatch.setattr(loom, "_several", True, raising=False)
    f(**tensors, **rest)
    for one in tensors:
        lib.args = None
        with pytest.raises(ValueError, match="cuda:1"):
            f(**{n: _elsewhere(t) if n == one else t for n, t in tensors.items()}, **rest)
        assert lib.args is None, one
    monkeypatch.setattr(loom, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError, match="current device"):
        f(**tensors, **rest)
    assert lib.args is None


@pytest.mark.parametrize("name", NAMES)
def test_a_flag_or_number_that_raises(loom, name):  # noqa: F811
    class Broken:
        def __bool__(self):
            raise KeyError("flag")

        __int__ = __float__ = __index__ = __bool__

    f, tensors, rest, _ = _calls(loom)[name]
    extra = {"chunk": "causal", "plan": "page_size", "axes": "interleaved", "axes_cache": "interleaved", "axes_bwd": "interleaved"}[name]
    with pytest.raises(KeyError, match="flag"):
        f(**tensors, **{**rest, extra: Broken()})
