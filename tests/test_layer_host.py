"""What the layer and its cache refuse on the host, before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2609_29219_gb300 import layer as layer_mod


def test_a_full_cache_is_refused():
    cache = layer_mod.PagedCache(2, 40, 1, 64, page=16, device="cpu")  # 3 pages a sequence
    first, slots = cache.take(40)
    assert first.tolist() == list(range(40)) * 2 and len(set(slots.tolist())) == 80
    with pytest.raises(ValueError, match="8"):
        cache.take(9)
    assert cache.lens.tolist() == [40, 40]  # nothing was taken
    pos, last = cache.take(8)
    assert pos.tolist() == list(range(40, 48)) * 2 and not set(last.tolist()) & set(slots.tolist())
    with pytest.raises(ValueError):
        cache.take(1)
    with pytest.raises(ValueError):
        cache.take(-1)


def test_a_step_past_the_rotation_tables_is_refused():
    layer = layer_mod.AttentionLayer(model=64, Hq=2, Hkv=1, D=64, positions=5, device="cpu")
    cache = layer_mod.PagedCache(2, 16, 1, 64, device="cpu")
    cache.take(5)
    with pytest.raises(ValueError, match="position 5"):
        layer.step(torch.zeros((2, 64), dtype=torch.bfloat16), cache)
    assert cache.used == 5 and cache.lens.tolist() == [5, 5]
