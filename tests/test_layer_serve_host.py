"""What a layer that serves requests refuses on the host, before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_2609_29219_gb300 import layer as layer_mod

X, NEW = torch.zeros((3, 64), dtype=torch.bfloat16), torch.tensor([2, 1], dtype=torch.int32)


@pytest.mark.parametrize("capacity,page,rows", [(41, 16, 48), (40, 16, 48), (41, 8, 48), (200, 8, 200)])
def test_a_cache_past_the_rotation_tables_is_refused(capacity, page, rows):
    """Its requests may grow to whole pages, and a position past the tables would be clamped to them."""
    layer = layer_mod.AttentionLayer(model=64, Hq=2, Hkv=1, D=64, positions=40, device="cpu")
    cache = layer_mod.RequestCache(2, 30, capacity, 1, 64, page=page, device="cpu")
    assert cache.capacity == rows
    with pytest.raises(ValueError, match=f"40 positions.* {rows} "):
        layer.serve(X, cache, NEW)


def test_a_cache_that_the_rotation_tables_reach():
    layer = layer_mod.AttentionLayer(model=64, Hq=2, Hkv=1, D=64, positions=48, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):  # the next thing that is wrong
        layer.serve(X, layer_mod.RequestCache(2, 30, 41, 1, 64, device="cpu"), NEW)
