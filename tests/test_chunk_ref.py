"""The 64-bit references of the chunk's attention and the step's bookkeeping, against other ways to the same."""
import math

import pytest

torch = pytest.importorskip("torch")

from tests import chunk_ref as ref  # noqa: E402


def test_attention_against_torch():
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 2, 8), (7, 8), (7, 8)))
    o, bo, lse, bl = ref.attention(q, k, v, True, 0.3)
    for i in range(3):
        n = 7 - 3 + i + 1
        s = q[i] @ k[:n].T * 0.3
        assert torch.allclose(o[i], torch.softmax(s, -1) @ v[:n]) and torch.allclose(lse[i], torch.logsumexp(s, -1))
    assert (bo > 0).all() and (bo < 0.05).all() and (bl < 1e-4).all()


def test_rows_that_see_nothing():
    q = torch.ones((3, 1, 8), dtype=torch.float64)
    k = torch.ones((2, 8), dtype=torch.float64)
    o, _, lse, _ = ref.attention(q, k, k, True, 1.0)
    assert (o[0] == 0).all() and lse[0, 0] == -math.inf and ((o[1:] - 1).abs() < 1e-14).all()


def test_gathered_pages():
    c = torch.arange(2 * 4 * 3 * 1.0).view(2, 4, 3, 1)
    got = ref.gathered(c, [1, 7, 0], 10, "nhd")
    assert got.shape == (10, 3, 1) and (got[:4] == c[1]).all() and (got[4:8] == 0).all() and (got[8:] == c[0, :2]).all()
    assert (ref.gathered(c.transpose(1, 2), [1, 0], 8, "hnd") == torch.cat((c[1], c[0]))).all()


def test_plan_by_hand():
    # pages of 4; request 0: 3 cached + 2 -> one more page; 1 is over and gives back 7 and 5; 2 asks for 3
    # pages, of which one is left after 0: refused; 3 needs none
    table = [[9, -1, -1], [7, 5, -1], [-1, -1, -1], [2, -1, -1]]
    cu, lens, pos, slots, granted, table, free, count = ref.plan([2, -1, 10, 1], [3, 6, 0, 2], table, [1] + [0] * 9, 1, 15, 4, 10)
    assert cu == [0, 2, 2, 12, 13] and lens == [5, 0, 0, 3] and granted == [2, 0, 0, 1]
    assert table[0] == [9, 5, -1] and table[2] == [-1, -1, -1] and free[:3] == [1, 7, 0] and count == 2
    assert pos == [3, 4] + [0] * 10 + [2, 0, 0] and slots == [39, 20] + [-1] * 10 + [10, -1, -1]
