"""Attention of a chunk of new tokens over a paged cache, against the formula in 64 bits (tests/chunk_ref.py)."""
import math

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


class Case:
    """Caches whose rows past a sequence's keys, and pages that are nobody's, are NaN; table entries past a
    sequence's pages are out of range."""

    def __init__(self, ql, kl, Hq, Hkv, D, page=16, layout="nhd", pad=0, seed=0, spread=1.0):
        import torch
        gen = torch.Generator().manual_seed(seed)
        per = [ref.pages(n, page) for n in kl]
        total = sum(per) + 2
        order = torch.randperm(total, generator=gen).to(torch.int32)
        self.table = torch.full((len(kl), max(per + [1]) + 1), 1 << 30, dtype=torch.int32)
        k, v = (torch.full((total, page, Hkv, D), math.nan, dtype=torch.bfloat16) for _ in range(2))
        at = 0
        for b, n in enumerate(kl):
            rows = order[at:at + per[b]]
            at += per[b]
            self.table[b, :per[b]] = rows
            for c in (k, v):
                x = torch.full((per[b] * page, Hkv, D), math.nan, dtype=torch.bfloat16)
                x[:n] = torch.randn((n, Hkv, D), generator=gen).bfloat16()
                c[rows.long()] = x.view(per[b], page, Hkv, D)
        self.k, self.v = ((x if layout == "nhd" else x.transpose(1, 2).contiguous()) for x in (k, v))
        self.q = (spread * torch.randn((sum(ql) + pad, Hq, D), generator=gen)).bfloat16()
        self.ql, self.kl, self.layout, self.D = ql, kl, layout, D
        self.cu = [sum(ql[:i]) for i in range(len(ql) + 1)]

    def device(self):
        import torch
        i32 = dict(dtype=torch.int32, device="cuda")
        return (self.q.cuda(), self.k.cuda(), self.v.cuda(), self.table.cuda(), torch.tensor(self.cu, **i32),
                torch.tensor(self.kl, **i32))

    def exact(self, causal, scale=None):
        return ref.chunk(self.q, self.k, self.v, self.table, self.cu, self.kl, causal, scale or self.D ** -0.5, self.layout)


def _check(got, lse, exact, what=""):
    import torch
    eo, bo, el, bl = exact
    real = ~torch.isnan(el[0])  # tokens that are some sequence's
    got, lse = got.double().cpu(), lse.double().cpu()
    over = (got[real] - eo[real]).abs() - bo[real]
    assert torch.isfinite(got[real]).all(), f"{what}: not finite"
    assert not (over > 0).any(), f"{what}: o past the bound by {float(over.max()):.3g}"
    lse, el, bl = lse[:, real], el[:, real], bl[:, real]
    assert torch.equal(torch.isinf(lse), torch.isinf(el)) and not torch.isnan(lse).any(), f"{what}: rows that see nothing"
    fin = torch.isfinite(el)
    over = (lse[fin] - el[fin]).abs() - bl[fin]
    assert not (over > 0).any(), f"{what}: lse past the bound by {float(over.max()):.3g}"


SHAPES = [  # new tokens, keys, Hq, Hkv, D, page, layout
    ([1], [1], 1, 1, 64, 8, "nhd"),
    ([1], [0], 4, 2, 128, 16, "hnd"),
    ([3], [2], 4, 2, 64, 16, "nhd"),
    ([0, 0, 5, 0], [7, 0, 5, 9], 8, 8, 128, 16, "nhd"),
    ([1] * 7, [1, 63, 64, 65, 127, 128, 129], 32, 8, 128, 16, "nhd"),
    ([2, 7, 4], [300, 7, 1000], 16, 2, 64, 32, "hnd"),
    ([130], [130], 32, 8, 128, 64, "nhd"),
    ([17, 300, 1], [300, 300, 1000], 28, 4, 128, 8, "hnd"),
    ([65, 64, 63], [65, 200, 64], 10, 2, 64, 192, "nhd"),
    ([200], [5000], 6, 3, 128, 128, "hnd"),
    ([1, 1], [20000, 3], 16, 2, 64, 16, "nhd"),
    ([600, 1, 1], [700, 900, 0], 5, 5, 64, 16, "nhd"),
    ([3, 2], [40, 500], 130, 1, 64, 16, "hnd"),
    ([9], [77], 131, 1, 128, 16, "nhd"),
    ([4, 33], [100, 50], 128, 1, 128, 16, "nhd"),
    ([33, 70], [200, 10], 48, 2, 64, 64, "hnd"),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("ql,kl,Hq,Hkv,D,page,layout", SHAPES)
def test_against_the_formula(loom, ql, kl, Hq, Hkv, D, page, layout, causal):
    c = Case(ql, kl, Hq, Hkv, D, page, layout)
    o, lse = loom.loom_attn_chunk_paged(*c.device(), causal=causal, layout=layout, return_lse=True)
    loom.loom_attn_check_error()
    _check(o, lse, c.exact(causal))


def test_many_sequences(loom):
    ql = [(7 * i) % 4 for i in range(700)]
    kl = [(37 * i) % 90 for i in range(700)]
    c = Case(ql, kl, 4, 2, 64)
    o, lse = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    _check(o, lse, c.exact(True))


def test_large_scores(loom):
    """Softmax rows that one key rules, and a running maximum that moves from tile to tile."""
    c = Case([40, 1], [900, 2000], 8, 2, 128, spread=20.0)
    o, lse = loom.loom_attn_chunk_paged(*c.device(), return_lse=True, scale=0.4)
    _check(o, lse, c.exact(True, 0.4))


def test_padding_is_left_alone(loom):
    import torch
    c = Case([5, 130], [60, 200], 8, 2, 128, pad=9)
    o, lse = torch.full_like(c.q, 7.0).cuda(), torch.full((8, 144), 3.0, device="cuda")
    r = loom.loom_attn_chunk_paged(*c.device(), o, lse)
    assert r[0] is o and r[1] is lse
    _check(o, lse, c.exact(True))
    assert (o[135:] == 7).all() and (lse[:, 135:] == 3).all()


def test_pages_that_there_are_not(loom):
    """Entries outside the cache read as zeros; a length past the table is cut to it."""
    import torch
    c = Case([3, 2], [100, 64], 4, 2, 64)
    c.table[0, 2], c.table[1, 1] = -5, c.k.shape[0]
    o, lse = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    _check(o, lse, c.exact(True))
    c = Case([2], [64], 4, 2, 64)
    c.table = c.table[:, :4].contiguous()
    c.kl = [1000]
    o, lse = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    _check(o, lse, c.exact(True))
    c.kl = [-3]
    o, lse = loom.loom_attn_chunk_paged(*c.device(), return_lse=True)
    assert (o == 0).all() and torch.isneginf(lse).all()


def test_a_sequence_reaches_no_other(loom):
    """NaN in one sequence's queries, keys and values stays there."""
    import torch
    c = Case([70, 70, 1], [200, 200, 300], 8, 2, 128)
    d = list(c.device())
    clean = loom.loom_attn_chunk_paged(*d)
    d[0][70:140] = math.nan
    for x in d[1:3]:
        x[c.table[1, :13].long().cuda()] = math.nan
    got = loom.loom_attn_chunk_paged(*d)
    assert torch.equal(got[:70], clean[:70]) and torch.equal(got[140:], clean[140:]) and torch.isnan(got[70:140]).all()


def test_caches_past_32_bits(loom):
    """Pages whose values lie past 2^32 elements from the cache's beginning."""
    import torch
    page, Hkv, D = 64, 8, 128
    num = (1 << 32) // (page * Hkv * D) + 40
    c = Case([40, 1], [300, 2000], 16, Hkv, D, page)
    d = list(c.device())
    for i in (1, 2):
        big = torch.empty((num, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
        big[-d[i].shape[0]:] = d[i]
        d[i] = big
    d[3] = torch.where(d[3] < c.k.shape[0], d[3] + num - c.k.shape[0], d[3])
    o, lse = loom.loom_attn_chunk_paged(*d, return_lse=True)
    _check(o, lse, c.exact(True))


def test_as_many_keys_as_there_may_be(loom):
    """2^31 - 64 keys, all of them one page's: its attention, and LSE that much larger.

    A CTA of at least 120 adds up to 2^31 / 128 / 120 = 139811 tiles: l in one addition each, off by half a step, o in
    eight, off by a step at most."""
    import torch
    most = (1 << 31) // 64 - 1
    c = Case([1], [64], 4, 1, 64, 64)
    d = list(c.device())
    d[3] = torch.full((1, most), int(c.table[0, 0]), dtype=torch.int32, device="cuda")
    d[5] = torch.full((1,), most * 64, dtype=torch.int32, device="cuda")
    o, lse = loom.loom_attn_chunk_paged(*d, return_lse=True)
    loom.loom_attn_check_error()
    eo, bo, el, bl = c.exact(True)
    rows = c.table[0, :1].tolist()
    p = torch.exp(torch.einsum("thd,kd->thk", c.q.double(), ref.gathered(c.k, rows, 64, "nhd")[:, 0]) / 8 - el.T[..., None])
    sizes = torch.einsum("thk,kd->thd", p, ref.gathered(c.v, rows, 64, "nhd")[:, 0].abs())
    tiles = 139811
    assert ((o.double().cpu() - eo).abs() <= bo + tiles * (8 * 2.0 ** -23 + 2.0 ** -24) * (sizes + eo.abs())).all()
    assert ((lse.double().cpu() - el - math.log(most)).abs() <= 2 * bl + tiles * 2.0 ** -24 * 1.1).all()


def test_a_key_that_is_nan_in_a_sequence_of_many_pieces(loom):
    """It is in one of the pieces that are joined, and in the row's LSE as in its output."""
    import torch
    c = Case([1, 1], [40000, 40000], 4, 1, 128)
    d = list(c.device())
    d[1][c.table[0, 1200].long().cuda(), 5] = math.nan
    o, lse = loom.loom_attn_chunk_paged(*d, return_lse=True)
    assert torch.isnan(o[0]).all() and torch.isnan(lse[:, 0]).all()
    assert torch.isfinite(o[1]).all() and torch.isfinite(lse[:, 1]).all()


SPLIT = [([1, 1, 1], [9000, 5000, 70], 32, 8, 128), ([300], [4000], 16, 2, 64), ([3, 400, 1], [3000, 400, 2000], 28, 4, 128)]


@pytest.mark.parametrize("ql,kl,Hq,Hkv,D", SPLIT)
def test_the_same_bits_whatever_the_workspace_held(loom, ql, kl, Hq, Hkv, D):
    import torch
    c = Case(ql, kl, Hq, Hkv, D)
    d = c.device()
    want = loom.loom_attn_chunk_paged(*d, return_lse=True)
    _check(*want, c.exact(True))
    n = loom.loom_attn_chunk_paged_workspace_bytes(len(ql), Hq, Hkv, sum(ql), D)
    for fill in (0, 1, 127, 255):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            got = loom.loom_attn_chunk_paged(*d, workspace=ws, return_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_one_workspace_for_calls_of_all_sizes(loom):
    import torch
    cases = [Case(ql, kl, Hq, Hkv, D, seed=i) for i, (ql, kl, Hq, Hkv, D) in enumerate(SPLIT)]
    ws = torch.empty(41 << 20, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        for c in cases:
            o, lse = loom.loom_attn_chunk_paged(*c.device(), workspace=ws, return_lse=True)
            _check(o, lse, c.exact(True))


def test_matches_the_decode_of_single_tokens(loom):
    """The same numbers as the paged decode, up to either's bound."""
    import torch
    c = Case([1] * 5, [1, 700, 64, 3000, 129], 32, 8, 128, seed=3)
    q, k, v, table, cu, lens = c.device()
    o, lse = loom.loom_attn_chunk_paged(q, k, v, table, cu, lens, return_lse=True)
    d, dl = loom.loom_attn_decode_paged(q.unsqueeze(2), k, v, table.clamp(max=k.shape[0]), lens, return_lse=True)
    _, bo, _, bl = c.exact(True)
    assert ((o.double() - d[:, :, 0].double()).abs().cpu() <= 2 * bo).all()
    assert ((lse.T.double() - dl.double()).abs().cpu() <= 2 * bl.T).all()


def test_captured_and_replayed_with_other_lengths(loom):
    """One graph serves every step whose sizes fit: the lengths are read on the device."""
    import torch
    Hq, Hkv, D, T, B = 16, 4, 128, 200, 4
    cases = [Case([100, 1, 60, 1], [2000, 300, 60, 77], Hq, Hkv, D, pad=38, seed=1),
             Case([1, 1, 1, 1], [900, 10, 1500, 4000], Hq, Hkv, D, pad=196, seed=2),
             Case([0, 200, 0, 0], [0, 800, 5, 0], Hq, Hkv, D, seed=3)]
    most, num = max(c.table.shape[1] for c in cases), max(c.k.shape[0] for c in cases)
    q = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((num, 16, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.zeros((B, most), dtype=torch.int32, device="cuda")
    cu, lens = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    loom.loom_attn_chunk_paged(q, k, v, table, cu, lens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o, lse = loom.loom_attn_chunk_paged(q, k, v, table, cu, lens, return_lse=True)
    for c in cases + cases:
        for to, x in zip((q, k, v, cu, lens), (c.device()[i] for i in (0, 1, 2, 4, 5))):
            to[:x.shape[0]] = x
        table[:, :c.table.shape[1]] = c.table.cuda()
        graph.replay()
        torch.cuda.synchronize()
        _check(o, lse, c.exact(True))


def test_on_a_stream_given(loom):
    import torch
    c = Case([40, 3], [900, 500], 16, 2, 64)
    d = c.device()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, lse = loom.loom_attn_chunk_paged(*d, stream=side, return_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    _check(o, lse, c.exact(True))


def test_two_streams_at_once(loom):
    import torch
    cases = [Case([1, 60], [6000, 3000], 16, 2, 64, seed=i) for i in range(2)]
    dev = [c.device() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    out = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                out[i].append(loom.loom_attn_chunk_paged(*dev[i], return_lse=True))
    torch.cuda.synchronize()
    for c, rs in zip(cases, out):
        exact = c.exact(True)
        for o, lse in rs:
            _check(o, lse, exact)


def test_refusals(loom):
    import torch
    q, k, v, table, cu, lens = Case([4, 3], [30, 20], 4, 2, 64).device()
    f = loom.loom_attn_chunk_paged
    with pytest.raises(TypeError, match="q must be"):
        f(q.float(), k, v, table, cu, lens)
    with pytest.raises(ValueError, match="contiguous"):
        f(q.transpose(0, 1), k, v, table, cu, lens)
    with pytest.raises(ValueError, match="one shape"):
        f(q, k, v[:1], table, cu, lens)
    with pytest.raises(ValueError, match="one shape"):
        f(q, k[..., :32].contiguous(), v[..., :32].contiguous(), table, cu, lens)
    with pytest.raises(ValueError, match="layout"):
        f(q, k, v, table, cu, lens, layout="dhn")
    with pytest.raises(ValueError, match="cu_seqlens_q"):
        f(q, k, v, table, cu[:2], lens)
    with pytest.raises(ValueError, match="seqlens_k"):
        f(q, k, v, table, cu, lens[:1])
    with pytest.raises(TypeError, match="seqlens_k must be"):
        f(q, k, v, table, cu, lens.long())
    with pytest.raises(ValueError, match="CUDA"):
        f(q, k, v, table.cpu(), cu, lens)
    with pytest.raises(ValueError, match="o must have"):
        f(q, k, v, table, cu, lens, q[:3].clone())
    with pytest.raises(ValueError, match="lse must be"):
        f(q, k, v, table, cu, lens, None, torch.zeros((7, 4), device="cuda"))
    with pytest.raises(loom.LoomError, match="WORKSPACE"):
        f(q, k, v, table, cu, lens, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(loom.LoomError, match="UNSUPPORTED"):
        f(q, k[:, :12].contiguous(), v[:, :12].contiguous(), table, cu, lens)
    with pytest.raises(loom.LoomError, match="INVALID"):
        f(q, k, v, table, cu, lens, scale=-1.0)
    assert f(q[:0], k, v, table, cu, lens).shape == (0, 4, 64)
