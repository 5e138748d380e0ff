"""How the backward pass deals its work, by its query (no GPU needed)."""
import pytest

from tests.test_abi_grad import lib  # noqa: F401


def _plan(lib, *sizes):  # noqa: F811
    import ctypes
    out = (ctypes.c_int * 4)(9, 9, 9, 9)
    return lib.loom_attn_bwd_plan(*sizes, out), list(out)


@pytest.mark.parametrize("sizes,expect", [
    ((0, 8, 2, 100, 100, 64, 0, 0), 1), ((1, 8, 3, 100, 100, 64, 0, 0), 1), ((1, 8, 2, 0, 100, 64, 0, 0), 1),
    ((1, 8, 2, 100, 99, 64, 1, 0), 1), ((1, 8, 2, 100, 100, 64, 2, 0), 1), ((1, 8, 2, 100, 100, 64, 0, 2), 1),
    ((1, 8, 2, -1, 100, 64, 0, 1), 1), ((1, 8, 2, 100, 100, 96, 0, 0), 2), ((1 << 20, 8, 2, 1 << 20, 1 << 20, 64, 0, 0), 2)])
def test_refusals(lib, sizes, expect):  # noqa: F811
    assert _plan(lib, *sizes) == (expect, [9, 9, 9, 9])


def test_refuses_no_place_for_the_plan(lib):  # noqa: F811
    assert lib.loom_attn_bwd_plan(1, 8, 2, 100, 100, 64, 0, 0, None) == 1


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [0, 1])
def test_shares_and_workspace_agree(lib, causal, D):  # noqa: F811
    """Whole items have no partial sums in the workspace; a share of an item has 128 rows of fp32 for each
    of its gradients."""
    status, (kv, q, kv_block, q_block) = _plan(lib, 2, 32, 32, 700, 700, D, causal, 0)
    assert (status, kv, q) == (0, 1, 1) and 1 <= kv_block <= 64 and 1 <= q_block <= 64
    stats = 64 * 6 * 1024
    assert lib.loom_attn_bwd_workspace_bytes(2, 32, 32, 700, 700, D) == 256 + stats
    status, (kv, q, _, _) = _plan(lib, 1, 4, 1, 1000, 4000, D, causal, 0)
    assert status == 0 and kv > 1 and q > 1
    assert lib.loom_attn_bwd_workspace_bytes(1, 4, 1, 1000, 4000, D) >= 32 * kv * 1024 * D + 32 * q * 512 * D
    # ragged: the totals; no blocks of planes
    status, (kv, q, kv_block, q_block) = _plan(lib, 1, 4, 1, 1000, 4000, D, causal, 1)
    assert status == 0 and kv > 1 and q > 1 and kv_block == q_block == 0
    assert _plan(lib, 3, 4, 1, 0, 0, D, causal, 1)[0] == 0
