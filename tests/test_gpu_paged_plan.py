"""A serving step's bookkeeping on the device, against the same request by request (tests/chunk_ref.py)."""
import random

import pytest

from tests import chunk_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loom():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_29219_gb300 as m
    return m


def _ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tables(rng, lens, most, page, spare):
    """Tables of pages dealt at random, the free list, and the pages in all."""
    held = [ref.pages(n, page) for n in lens]
    num = sum(held) + spare
    order = list(range(num))
    rng.shuffle(order)
    table = [[-1] * most for _ in lens]
    for row, n in zip(table, held):
        for j in range(n):
            row[j] = order.pop()
    return table, order + [0] * (num - spare), num


def _check(loom, new, lens, table, free, count, T, page, num, in_place=False):
    import torch
    want = ref.plan(new, lens, table, free, count, T, page, num)
    tn, tl, tt, tf, tc = (_ints(x) for x in (new, lens, table, free, [count]))
    if in_place:
        got = loom.loom_paged_plan(tn, tl, tt, tf, tc, T, page, seqlens_k=tl)
        assert got[1] is tl
    else:
        out = _ints([77])
        got = loom.loom_paged_plan(tn, tl, tt, tf, tc, T, page, free_count_out=out)
        assert int(tc) == count and torch.equal(tl, _ints(lens))
        tc = out
    for g, w, name in zip((*got, tt, tf), want[:7], ("cu", "seqlens", "positions", "slots", "granted", "table", "free")):
        assert torch.equal(g, _ints(w).view(g.shape)), name
    assert int(tc) == want[7]
    return want


SIZES = [  # requests, most new tokens, most cached, page, of how many one is over, free pages more than needed, padding
    (1, 1, 0, 16, 0, 1, 0), (1, 300, 70, 8, 0, 50, 5), (4, 1, 100, 16, 0, 10, 0), (33, 50, 200, 16, 5, 500, 7),
    (33, 50, 200, 16, 5, 40, 7), (33, 50, 200, 16, 3, 0, 0), (300, 40, 90, 64, 20, 20, 3000), (1025, 3, 50, 8, 7, 900, 1),
    (1300, 9, 300, 1, 9, 3000, 0), (8192, 2, 40, 16, 11, 3000, 100), (5, 3000, 5000, 128, 0, 200, 0)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,n,l,page,over,spare,pad", SIZES)
def test_against_request_by_request(loom, B, n, l, page, over, spare, pad, in_place):
    rng = random.Random(B + spare)
    lens = [rng.randint(0, l) for _ in range(B)]
    new = [-rng.randint(1, 9) if over and rng.randrange(over) == 0 else rng.randint(0, n) for _ in range(B)]
    most = ref.pages(n + l, page)
    table, free, num = _tables(rng, lens, most, page, spare)
    _check(loom, new, lens, table, free, spare, sum(max(x, 0) for x in new) + pad, page, num, in_place)


def test_refused_for_the_table_and_for_the_tokens(loom):
    table, free, num = _tables(random.Random(3), [30, 0, 30, 5], 2, 16, 10)
    want = _check(loom, [3, 32, 2, 9], [30, 0, 30, 5], table, free, 10, 100, 16, num)
    assert want[4] == [0, 32, 2, 9]
    want = _check(loom, [3, 32, 2, 0], [20, 0, 30, 5], table, free, 10, 36, 16, num)
    assert want[4] == [3, 32, 0, 0] and want[0] == [0, 3, 35, 36, 36]
    _check(loom, [3, 32, 2, 9], [30, 0, 30, 5], table, free, 10, 0, 16, num)


def test_as_many_tokens_as_there_may_be(loom):
    T = (1 << 31) - 1
    table, free = _ints([[0] * 4]), _ints(range(4))
    cu, _, positions, slots, granted = loom.loom_paged_plan(_ints([20]), _ints([0]), table, free, _ints([4]), T, 16)
    assert cu.tolist() == [0, 20] and granted.tolist() == [20] and positions[:20].tolist() == list(range(20))
    assert slots[:20].tolist() == [3 * 16 + i for i in range(16)] + [2 * 16 + i for i in range(4)]
    for at in (20, 1 << 30, T - 70000):  # (the largest step's ends and one in its middle)
        assert (slots[at:at + 70000] == -1).all() and (positions[at:at + 70000] == 0).all()


def test_every_page_is_given_back(loom):
    lens = [40, 0, 17, 64]
    table, free, num = _tables(random.Random(4), lens, 6, 16, 3)
    want = _check(loom, [-1] * 4, lens, table, free, 3, 5, 16, num)
    assert want[7] == num and sorted(want[6]) == list(range(num))
    # pages given back are the first to be taken
    want = _check(loom, [-1, 20, 30, 1], lens, table, free, 3, 60, 16, num)
    assert want[5][1][:2] == [want[5][0][2], want[5][0][1]]


def test_numbers_out_of_range(loom):
    """Lengths outside the table's row, a free count outside the list, pages that there are not, lengths past 2^31 in
    sum; nothing outside the buffers is read or written."""
    import torch
    table, free, num = _tables(random.Random(5), [20, 20, 20], 4, 16, 6)
    _check(loom, [1, 1, 1], [-7, 1 << 30, 20], table, free, 6, 3, 16, num)
    _check(loom, [1, 50, -1], [20, 0, 20], table, free, 1 << 30, 51, 16, num)
    _check(loom, [1, 50, 1], [20, 0, 20], table, free, -4, 52, 16, num)
    big = (1 << 31) - 1
    _check(loom, [big, big, 2], [20, 20, 20], table, free, 6, 40, 16, num)
    table[0][0], table[0][1] = num, -3
    _check(loom, [5, 0, 1], [20, 20, 20], table, free, 6, 6, 16, num)
    # one page in two tables: the list is cut at its length
    lens, t = _ints([64, 64, 64]), _ints([[0, 1, 2, 3]] * 3)
    f, c = torch.zeros(6, dtype=torch.int32, device="cuda"), _ints([0])
    loom.loom_paged_plan(_ints([-1, -1, -1]), lens, t, f, c, 0, 16)
    assert int(c) == 6 and f.tolist() == [0, 1, 2, 3, 0, 1]


def test_steps_captured_and_replayed(loom):
    """A graph that plans in place runs a server's steps: prompts, next tokens, ends."""
    import torch
    rng = random.Random(8)
    B, page, most, num, T = 6, 16, 8, 30, 64
    new, lens, table = _ints([0] * B), _ints([0] * B), _ints([[-1] * most] * B)
    free, count = _ints(list(range(num))), _ints([num])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    loom.loom_paged_plan(new, lens, table, free, count, T, page, seqlens_k=lens)
    with torch.cuda.graph(graph, stream=side):
        got = loom.loom_paged_plan(new, lens, table, free, count, T, page, seqlens_k=lens)
    state = ([0] * B, table.tolist(), free.tolist(), num)
    for _ in range(40):
        n = [rng.choice((1, 1, 1, 0, 20, 33)) if x < 90 else -1 for x in state[0]]
        want = ref.plan(n, state[0], state[1], state[2], state[3], T, page, num)
        new.copy_(_ints(n))
        graph.replay()
        for g, w in zip(got, want[:5]):
            assert g.tolist() == w
        assert table.tolist() == want[5] and int(count) == want[7] and free.tolist()[:want[7]] == want[6][:want[7]]
        held = [p for r, l in zip(want[5], want[1]) for p in r[:ref.pages(l, page)]]
        assert sorted(held + want[6][:want[7]]) == list(range(num))
        state = want[1], want[5], want[6], want[7]


def test_refusals(loom):
    import torch
    n, l, t, f, c = _ints([1, 1]), _ints([3, 3]), _ints([[0, -1], [1, -1]]), _ints([2, 3, 0, 0]), _ints([2])
    g = loom.loom_paged_plan
    with pytest.raises(TypeError, match="lens must be"):
        g(n, l.long(), t, f, c, 2, 16)
    with pytest.raises(ValueError, match="new_lens must be a CUDA"):
        g(n.cpu(), l, t, f, c, 2, 16)
    with pytest.raises(ValueError, match="block_table must have 2"):
        g(n, l, t[0], f, c, 2, 16)
    with pytest.raises(ValueError, match="must be"):
        g(n, l[:1], t, f, c, 2, 16)
    with pytest.raises(ValueError, match="num_tokens"):
        g(n, l, t, f, c, -1, 16)
    with pytest.raises(ValueError, match="slots must be"):
        g(n, l, t, f, c, 2, 16, slots=torch.zeros(3, dtype=torch.int32, device="cuda"))
    with pytest.raises(loom.LoomError, match="INVALID"):
        g(n, l, t, f, c, 2, 0)
