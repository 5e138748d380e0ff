"""A layer that serves requests: what its caller learns of those that the cache had no room for, and what a call that
is refused leaves behind."""
import pytest

from tests.test_gpu_given_stream import loom  # noqa: F401

pytestmark = pytest.mark.gpu


def _ints(*x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _layer():
    from paper_2609_29219_gb300 import layer as mod
    return mod, mod.AttentionLayer(model=128, Hq=4, Hkv=2, D=64, positions=64, seed=3)


def _held(cache):
    return cache.lens.tolist(), cache.table.tolist(), cache.free_pages[:int(cache.free_count)].tolist()


def test_a_request_without_room_is_told(loom):  # noqa: F811
    import torch
    mod, layer = _layer()
    x = torch.randn((30, 128), device="cuda").bfloat16()
    cache, alone = mod.RequestCache(3, 2, 64, 2, 64), mod.RequestCache(1, 4, 64, 2, 64)  # two pages: three requests want one each
    y = layer.serve(x, cache, _ints(10, 8, 12))
    assert cache.granted.tolist() == [10, 8, 0] and cache.lens.tolist() == [10, 8, 0]
    assert torch.equal(y[:10], layer.serve(x[:10].contiguous(), alone, _ints(10))) and alone.granted.tolist() == [10]
    layer.serve(x, cache, _ints(-1, 3, 12))  # the first one ends: there is room
    assert cache.granted.tolist() == [0, 3, 12] and cache.lens.tolist() == [0, 11, 12]
    loom.loom_attn_check_error()


def test_what_was_granted_after_a_replay(loom):  # noqa: F811
    """`granted` is of the last step, whether it was run or replayed, and whatever ran in between."""
    import torch
    mod, layer = _layer()
    x, new, cache = torch.randn((20, 128), device="cuda").bfloat16(), _ints(0, 0), mod.RequestCache(2, 1, 64, 2, 64)
    layer.serve(x, cache, new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.serve(x, cache, new)
    layer.serve(x, cache, _ints(7, 8))
    assert cache.granted.tolist() == [7, 0]
    new.copy_(_ints(9, 5))
    graph.replay()
    assert cache.granted.tolist() == [9, 0]
    new.copy_(_ints(-1, 5))
    graph.replay()
    assert cache.granted.tolist() == [0, 5] and cache.lens.tolist() == [0, 5]


def test_a_plan_of_its_own_keeps_its_grants(loom):  # noqa: F811
    """What `plan` returns is that call's, whatever comes after; `granted` is the layer's."""
    import torch
    mod, layer = _layer()
    cache = mod.RequestCache(2, 4, 64, 2, 64)
    first, second = cache.plan(_ints(5, 6), 11)[3], cache.plan(_ints(1, 0), 1)[3]
    layer.serve(torch.randn((8, 128), device="cuda").bfloat16(), cache, _ints(0, 8))
    third = cache.plan(_ints(2, 2), 4)[3]
    assert [t.tolist() for t in (first, second, third, cache.granted)] == [[5, 6], [1, 0], [2, 2], [0, 8]]


def test_a_plan_with_granted_given(loom, monkeypatch):  # noqa: F811
    """The compiled binding writes into it, as the Python code does, and takes no other shape or type."""
    import torch
    def run(granted):
        return loom.loom_paged_plan(_ints(3, 9, -1), _ints(0, 0, 4), table.clone(), free.clone(), _ints(1), 12, 16, granted=granted)
    table, free = torch.zeros((3, 2), dtype=torch.int32, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda")
    ways = [loom._fast, None]
    for fast in ways:
        monkeypatch.setattr(loom, "_fast", fast)
        out = _ints(7, 7, 7)
        r = run(out)
        assert r[4] is out and out.tolist() == [3, 9, 0] and all(torch.equal(a, b) for a, b in zip(r, run(None)))
        with pytest.raises(ValueError, match="granted must be"):
            run(_ints(7, 7))
        with pytest.raises(TypeError, match="granted must be"):
            run(out.long())


REFUSED = {  # what serve is given -> what it says
    "width": (lambda x, c: (x[:, :64].contiguous(), c), "model"), "rank": (lambda x, c: (x[0], c), "model"),
    "type": (lambda x, c: (x.float(), c), "bfloat16"), "rows": (lambda x, c: (x[::2], c), "contiguous"),
    "empty and of another width": (lambda x, c: (x[:0, :64], c), "model"),
    "cache of other heads": (lambda x, c: (x, _other(c, 1, 64)), "heads"), "cache of wider heads": (lambda x, c: (x, _other(c, 2, 128)), "heads")}


def _other(cache, Hkv, D):
    cache.k, cache.v = (t.new_zeros((*t.shape[:2], Hkv, D)) for t in (cache.k, cache.v))
    return cache


@pytest.mark.parametrize("name", REFUSED)
def test_a_call_that_is_refused_leaves_the_cache_alone(loom, name):  # noqa: F811
    import torch
    mod, layer = _layer()
    x, cache = torch.randn((20, 128), device="cuda").bfloat16(), mod.RequestCache(2, 8, 64, 2, 64)
    layer.serve(x, cache, _ints(9, 4))
    before = _held(cache)
    change, says = REFUSED[name]
    with pytest.raises((ValueError, TypeError), match=says):
        layer.serve(*change(x, cache), _ints(9, 4))
    assert _held(cache) == before


def test_a_step_without_tokens(loom):  # noqa: F811
    """Requests may end in a step that brings nothing else."""
    import torch
    mod, layer = _layer()
    x, cache = torch.randn((20, 128), device="cuda").bfloat16(), mod.RequestCache(2, 8, 64, 2, 64)
    layer.serve(x, cache, _ints(16, 4))
    y = layer.serve(x[:0], cache, _ints(-1, 0))
    loom.loom_attn_check_error()
    assert y.shape == (0, 128) and y.dtype == x.dtype and y.is_cuda
    assert cache.lens.tolist() == [0, 4] and int(cache.free_count) == 7
