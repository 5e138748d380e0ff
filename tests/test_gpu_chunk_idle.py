"""Attention of new tokens where few of many sequences bring any: the same bits as without the others."""
import pytest

from tests.test_gpu_chunk import Case, _check, loom  # noqa: F401

pytestmark = pytest.mark.gpu


def _among(c, rows, B):
    """The case's device tensors with its sequences at these rows of B, in order.  The others bring no token, but
    have keys (in pages that there are not)."""
    import torch
    q, k, v, table, cu, lens = c.device()
    at = torch.tensor(rows, device="cuda")
    wide = torch.full((B, table.shape[1]), 1 << 30, dtype=torch.int32, device="cuda")
    keys, tokens = (torch.full((B,), n, dtype=torch.int32, device="cuda") for n in (9, 0))
    wide[at], keys[at], tokens[at] = table, lens, cu.diff()
    return q, k, v, wide, torch.cat((cu[:1], tokens.cumsum(0).to(torch.int32))), keys


@pytest.mark.parametrize("rows,B", [
    ([0, 1], 3000), ([2998, 2999], 3000), ([0, 2999], 3000), ([5, 261], 262), ([5, 262], 263), ([5, 263], 264), ([383, 384], 400),
    ([0, 2, 4, 35, 67, 100, 355, 611, 868, 3000], 3300),
    ([300 * i + 7 * (i % 5) for i in range(60)], 20000)])
@pytest.mark.parametrize("D", [64, 128])
def test_few_of_many(loom, rows, B, D):  # noqa: F811
    import torch
    n = len(rows)
    c = Case([(1, 3, 70, 1, 20)[i % 5] for i in range(n)], [(500, 3, 90, 129, 1)[i % 5] for i in range(n)], 8, 4, D)
    want = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    _check(*want, c.exact(True))
    got = loom.loom_attn_chunk_paged(*_among(c, rows, B), return_lse=True)
    loom.loom_attn_check_error()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows", [[0, 1], [0, (1 << 20) - 1], [(1 << 20) - 2, (1 << 20) - 1]])
def test_a_million_rows_hold_nobody_up(loom, rows):  # noqa: F811
    """No wait inside the kernel lasts as long as a walk of the rows one by one does (75 ns a row)."""
    import torch
    c = Case([1, 1], [100, 900], 4, 2, 64, page=64)
    d = _among(c, rows, 1 << 20)
    want = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    loom.loom_debug_set_timeout_ns(20_000_000)
    try:
        got = loom.loom_attn_chunk_paged(*d, return_lse=True)
        loom.loom_attn_check_error()
    finally:
        loom.loom_debug_set_timeout_ns(0)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
