"""Serving calls with tensors whose sizes do not fit the C call's 32 bits: refused, not cut."""
import pytest

from tests.test_gpu_chunk import Case, loom  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["table", "free"])
@pytest.mark.parametrize("size", [(1 << 31) + 16, (1 << 32) + 16])
def test_sizes_past_32_bits(loom, name, size):  # noqa: F811
    """(2^32 + 16 entries of a row would be 16: no more than 256 of the sequence's keys.)"""
    import torch
    need = 4 * size + (2 << 30)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip(f"needs {need >> 30} GB")
    i32 = dict(dtype=torch.int32, device="cuda")
    big = torch.empty(size, **i32)  # (not filled: nothing reads it)
    one = lambda x: torch.full((1,), x, **i32)  # noqa: E731
    if name == "table":
        q, k, v, _, cu, lens = Case([1], [300], 4, 2, 64).device()
        with pytest.raises(loom.LoomError, match="UNSUPPORTED"):
            loom.loom_attn_chunk_paged(q, k, v, big.view(1, size), cu, lens)
        with pytest.raises(loom.LoomError, match="UNSUPPORTED"):
            loom.loom_paged_plan(one(1), one(0), big.view(1, size), torch.arange(4, **i32), one(4), 1, 16)
    else:
        with pytest.raises(loom.LoomError, match="UNSUPPORTED"):
            loom.loom_paged_plan(one(1), one(0), torch.zeros((1, 4), **i32), big, one(4), 1, 16)
