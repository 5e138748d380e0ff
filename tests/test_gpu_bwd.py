"""Attention's backward pass against the formulas in 64 bits, within bounds derived from its
roundings (tests/grad_ref.py)."""
import pytest

from tests import grad_ref as ref

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


def _normal(gen, *shape):
    import torch
    return torch.randn(shape, generator=gen).bfloat16()


def _check(got, exact, bound, what):
    import torch
    got = got.double().cpu()
    assert got.shape == exact.shape and torch.isfinite(got).all(), what
    over = (got - exact).abs() - bound
    assert not (over > 0).any(), f"{what}: {int((over > 0).sum())} of {over.numel()} past the bound, worst {float(over.max()):.3g}"


def _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, dlse, seed=0, scale=None, amp=1.0):
    """Forward and backward on the device, and the host's copies of what went in."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    q, k, v = amp * _normal(gen, B, Hq, Sq, D), _normal(gen, B, Hkv, Skv, D), _normal(gen, B, Hkv, Skv, D)
    do = _normal(gen, B, Hq, Sq, D)
    dl = torch.randn((B, Hq, Sq), generator=gen) if dlse else None
    dev = [t.cuda() for t in (do, q, k, v)]
    if causal and Sq > Skv:
        raise AssertionError("no such call")
    o, lse = loom.loom_attn_fwd(*dev[1:], causal=causal, scale=scale, return_lse=True)
    grads = loom.loom_attn_bwd(*dev, o, lse, causal=causal, scale=scale, dlse=None if dl is None else dl.cuda())
    loom.loom_attn_check_error()
    return (do, q, k, v, o.cpu(), lse.cpu(), dl), grads


def _check_dense(host, grads, causal, scale):
    do, q, k, v, o, lse, dl = [None if t is None else t.double() for t in host]
    for b in range(q.shape[0]):
        exact, bound = ref.attention_grads(do[b], q[b], k[b], v[b], o[b], lse[b], None if dl is None else dl[b], causal, scale)
        for g, e, bd, n in zip(grads, exact, bound, ("dq", "dk", "dv")):
            _check(g[b], e, bd, f"{n} of batch {b}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv", [
    (1, 1, 1, 1, 1), (1, 2, 1, 1, 300), (2, 2, 2, 128, 128), (1, 4, 1, 129, 129), (1, 3, 3, 127, 255), (2, 6, 2, 300, 411),
    (1, 8, 1, 64, 640), (1, 2, 2, 513, 513), (5, 2, 1, 3, 5), (1, 4, 4, 256, 256), (1, 1, 1, 131, 1000)])
def test_dense_against_the_formula(loom, B, Hq, Hkv, Sq, Skv, D, causal):
    host, grads = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, dlse=Sq % 2 == 1)
    _check_dense(host, grads, causal, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Sq,Skv", [(300, 100), (129, 1)])
def test_more_queries_than_keys(loom, Sq, Skv, D):
    host, grads = _dense(loom, 1, 4, 2, Sq, Skv, D, False, True)
    _check_dense(host, grads, False, D ** -0.5)


@pytest.mark.parametrize("causal", [False, True])
def test_many_items_and_a_scale_of_ones_own(loom, causal):
    """More items than CTAs, so that CTAs take several; sharp probabilities."""
    host, grads = _dense(loom, 3, 24, 8, 400, 400, 64, causal, False, scale=0.25, amp=2.0)
    _check_dense(host, grads, causal, 0.25)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv", [(1, 8, 1, 700, 700), (1, 2, 2, 1100, 1500), (1, 3, 1, 130, 2000), (2, 4, 1, 1000, 1000)])
def test_few_long_items_are_split(loom, B, Hq, Hkv, Sq, Skv, D, causal):
    """Few tiles with many steps, whose sums are split and joined (the workspace shows that they are);
    the same bits each time."""
    import torch
    host, grads = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, False)
    stats = B * Hq * Sq * 8
    assert loom.loom_attn_bwd_workspace_bytes(B, Hq, Hkv, Sq, Skv, D) > 4 * stats
    _check_dense(host, grads, causal, D ** -0.5)
    again = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, False)[1]
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


def _ragged(loom, ql, kl, Hq, Hkv, D, causal, dlse, seed=0, spoil=None):
    import torch
    gen = torch.Generator().manual_seed(seed)
    tq, tk = sum(ql), sum(kl)
    q, k, v, do = _normal(gen, tq, Hq, D), _normal(gen, tk, Hkv, D), _normal(gen, tk, Hkv, D), _normal(gen, tq, Hq, D)
    dl = torch.randn((Hq, tq), generator=gen) if dlse else None
    cq, ck = [torch.tensor([0] + list(x)).cumsum(0).to(torch.int32) for x in (ql, kl)]
    # O and LSE in 64 bits, as the forward pass returns them
    o, lse = torch.zeros(tq, Hq, D), torch.full((Hq, tq), -float("inf"))
    for b in range(len(ql)):
        a, e, c, d = int(cq[b]), int(cq[b + 1]), int(ck[b]), int(ck[b + 1])
        if e > a and d > c:
            x, y = ref.attention(q[a:e].transpose(0, 1).double(), k[c:d].transpose(0, 1).double(), v[c:d].transpose(0, 1).double(),
                                 causal, D ** -0.5)
            o[a:e], lse[:, a:e] = x.transpose(0, 1).float(), y.float()
    o = o.bfloat16()
    if spoil is not None:  # a sequence's own rows are no number or infinite
        a, e, c, d = int(cq[spoil]), int(cq[spoil + 1]), int(ck[spoil]), int(ck[spoil + 1])
        q[a:e], do[a:e], o[a:e], lse[:, a:e] = float("nan"), float("inf"), float("nan"), float("nan")
        k[c:d], v[c:d] = float("inf"), float("nan")
    host = (do, q, k, v, o, lse, dl)
    dev = [None if t is None else t.cuda() for t in host]
    grads = loom.loom_attn_bwd_varlen(*dev[:6], cq.cuda(), ck.cuda(), max(ql), max(kl), causal=causal, dlse=dev[6])
    loom.loom_attn_check_error()
    return host, grads, cq.tolist(), ck.tolist()


def _check_ragged(host, grads, cq, ck, causal, scale, skip=None):
    do, q, k, v, o, lse, dl = [None if t is None else t.double() for t in host]
    T = lambda t, a, e: t[a:e].transpose(0, 1)  # noqa: E731
    for b in range(len(cq) - 1):
        a, e, c, d = cq[b], cq[b + 1], ck[b], ck[b + 1]
        if b == skip:
            continue
        exact, bound = ref.attention_grads(T(do, a, e), T(q, a, e), T(k, c, d), T(v, c, d), T(o, a, e), lse[:, a:e],
                                           None if dl is None else dl[:, a:e], causal, scale)
        for g, (x, y), ex, bd, n in zip(grads, ((a, e), (c, d), (c, d)), exact, bound, ("dq", "dk", "dv")):
            if y > x:
                _check(g[x:y].transpose(0, 1), ex, bd, f"{n} of sequence {b}")


RAGGED = [
    ((100, 1, 300, 128, 129), None),               # lengths of one, a tile, a tile and one
    ((0, 77, 0, 200, 0), None),                    # empty sequences at both ends and between
    ((5, 200, 130), (260, 40, 130)),               # more queries than keys: rows that see nothing
    ((0, 150, 64, 10), (90, 0, 300, 7)),           # queries without keys, keys without queries
    ((3,) * 40, None),                             # many short ones
    ((1, 900, 700), None),                         # few long ones: split sums, shares without steps
    ((2, 5, 1200), (900, 1500, 3)),                # ... and rows that see nothing
]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,kl", RAGGED)
def test_ragged_against_the_formula(loom, ql, kl, causal, D):
    host, grads, cq, ck = _ragged(loom, ql, kl or ql, 6, 3, D, causal, len(ql) % 2 == 1)
    _check_ragged(host, grads, cq, ck, causal, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kl,ql", [((130, 130), (0, 150)), ((0, 140), (150, 150))])
def test_items_without_steps_between_others(loom, kl, ql, D):
    """Sequences without queries (or keys) in turn with others, several items for each CTA."""
    host, grads, cq, ck = _ragged(loom, ql * 30, kl * 30, 16, 16, D, False, False)
    _check_ragged(host, grads, cq, ck, False, D ** -0.5)
    for b in range(0, 60, 2):
        assert (grads[0][cq[b]:cq[b + 1]] == 0).all() and (grads[1][ck[b]:ck[b + 1]] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_a_sequence_of_nan_and_infinity_reaches_no_other(loom, causal, D):
    ql, kl = (70, 130, 200, 33), (70, 200, 190, 33)
    for spoil in (1, 2, 3):
        clean = _ragged(loom, ql, kl, 4, 2, D, causal, False)[1]
        host, grads, cq, ck = _ragged(loom, ql, kl, 4, 2, D, causal, False, spoil=spoil)
        _check_ragged(host, grads, cq, ck, causal, D ** -0.5, skip=spoil)
        for g, x, at in zip(grads, clean, (cq, ck, ck)):
            assert (g[:at[spoil]] == x[:at[spoil]]).all() and (g[at[spoil + 1]:] == x[at[spoil + 1]:]).all()


def test_rows_that_see_nothing_have_zero_gradients(loom):
    host, (dq, dk, dv), cq, ck = _ragged(loom, (300,), (40,), 2, 1, 64, True, True)
    assert (dq[:260] == 0).all() and (dq[261:] != 0).any()
    _, (dq, dk, dv), _, _ = _ragged(loom, (0, 20), (30, 20), 2, 1, 64, False, False)
    assert (dk[:30] == 0).all() and (dv[:30] == 0).all()


def test_no_queries_or_no_keys_at_all(loom):
    import torch
    mk = lambda n, h: torch.randn((n, h, 64), device="cuda").bfloat16()  # noqa: E731
    cu = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, k = mk(0, 4), mk(30, 2)
    lse = torch.zeros((4, 0), device="cuda")
    dq, dk, dv = loom.loom_attn_bwd_varlen(q, q, k, k, q, lse, cu(0, 0), cu(0, 30), 0, 30)
    assert dq.shape == (0, 4, 64) and (dk == 0).all() and (dv == 0).all()
    q, k = mk(30, 4), mk(0, 2)
    lse = torch.full((4, 30), -float("inf"), device="cuda")
    dq, dk, dv = loom.loom_attn_bwd_varlen(q, q, k, k, torch.zeros_like(q), lse, cu(0, 30), cu(0, 0), 30, 0)
    assert (dq == 0).all() and dk.shape == (0, 2, 64)
    loom.loom_attn_check_error()


@pytest.mark.parametrize("D", [64, 128])
def test_gradients_against_differences_of_the_loss(loom, D):
    """<gradient, u> of the kernels against central differences of the loss in 64 bits."""
    import torch
    host, grads = _dense(loom, 1, 4, 2, 150, 170, D, True, True, seed=3)
    do, q, k, v, _, _, dl = [t.double()[0] for t in host]
    scale = D ** -0.5

    def loss(q, k, v):
        o, lse = ref.attention(q, k, v, True, scale)
        return (do * o).sum() + (dl * lse).sum()

    o, lse = ref.attention(q, k, v, True, scale)
    _, bound = ref.attention_grads(do, q, k, v, o, lse, dl, True, scale)
    gen = torch.Generator().manual_seed(4)
    h = 1e-4
    for i, x in enumerate((q, k, v)):
        u = torch.randn(x.shape, generator=gen, dtype=torch.float64)
        at = lambda e: loss(*[y + e * u if j == i else y for j, y in enumerate((q, k, v))])  # noqa: E731
        slope = (at(h) - at(-h)) / (2 * h)
        got = (grads[i][0].double().cpu() * u).sum()
        # The kernel's roundings, and delta: O is rounded to bf16, which shifts each row's delta by up
        # to 2^-8 sum |dO| |O| and dS by P times that.
        shift = ref.BF16 * (do.abs() * o.abs()).sum(-1)
        ke = k.repeat_interleave(2, 0)
        s = (scale * q @ ke.transpose(1, 2)).masked_fill(~ref.seen_mask(150, 170, True), -float("inf"))
        p = torch.exp(s - lse[..., None]) * shift[..., None] * scale
        moved = (p @ ke.abs(), (p.transpose(1, 2) @ q.abs()).view(2, 2, 170, D).sum(1), torch.zeros_like(v))[i]
        assert abs(got - slope) <= ((bound[i] + moved) * u.abs()).sum() + 1e-5 * (grads[i][0].double().cpu().abs() * u.abs()).sum()


@pytest.mark.parametrize("causal", [False, True])
def test_the_same_inputs_give_the_same_bits(loom, causal):
    import torch
    a = _dense(loom, 2, 16, 4, 700, 700, 128, causal, False)[1]
    b = _dense(loom, 2, 16, 4, 700, 700, 128, causal, False)[1]
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_given_outputs_workspace_and_stream(loom):
    """Outputs and workspace of the caller's, whose contents do not matter, on a stream of its own,
    and replayed from a graph."""
    import torch
    B, Hq, Hkv, S, D = 1, 4, 2, 260, 128
    host, want = _dense(loom, B, Hq, Hkv, S, S, D, True, False)
    dev = [t.cuda() for t in host[:6]]
    need = loom.loom_attn_bwd_workspace_bytes(B, Hq, Hkv, S, S, D)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        outs = [torch.full_like(t, float("nan")) for t in dev[1:4]]
        got = loom.loom_attn_bwd(*dev, *outs, ws, causal=True)
    side.synchronize()
    assert all(x is y for x, y in zip(got, outs)) and all(torch.equal(x, y) for x, y in zip(got, want))
    with torch.cuda.stream(side):  # given as an argument, the current stream being another
        pass
    for t in outs:
        t.fill_(float("nan"))
    torch.cuda.synchronize()
    loom.loom_attn_bwd(*dev, *outs, ws, causal=True, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loom.loom_attn_bwd(*dev, *outs, ws, causal=True)
    for t in outs:
        t.fill_(float("nan"))
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
    loom.loom_attn_check_error()


def test_outputs_aligned_to_16_bytes_only(loom):
    import torch
    host, want = _dense(loom, 1, 4, 2, 260, 260, 64, True, False)
    dev = [t.cuda() for t in host[:6]]
    outs = [torch.empty(t.numel() + 8, dtype=torch.bfloat16, device="cuda")[8:].view(t.shape) for t in dev[1:4]]
    assert all(t.data_ptr() % 32 == 16 for t in outs)
    loom.loom_attn_bwd(*dev, *outs, causal=True)
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_offsets_past_32_bits(loom):
    """A packed batch of more than 2^31 values: its last sequence against a call of its own."""
    import torch
    H, D, n, last = 32, 128, 530_000, 333
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    gen = torch.Generator(device="cuda").manual_seed(5)
    mk = lambda: torch.randn((n + last, H, D), generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    q, k, v, do = mk(), mk(), mk(), mk()
    # sequences of one token, then the last
    ends = list(range(0, n, 4000)) + [n, n + last]
    cu = torch.tensor(ends, dtype=torch.int32, device="cuda")
    o, lse = torch.zeros_like(q), torch.full((H, n + last), 50.0, device="cuda")
    tail = [t[n:].contiguous() for t in (do, q, k, v)]
    cl = torch.tensor([0, last], dtype=torch.int32, device="cuda")
    ot, lt = loom.loom_attn_fwd_varlen(*tail[1:], cl, cl, last, causal=True, return_lse=True)
    o[n:], lse[:, n:] = ot, lt
    got = loom.loom_attn_bwd_varlen(do, q, k, v, o, lse, cu, cu, 4000, 4000, causal=True)
    want = loom.loom_attn_bwd_varlen(*tail, ot, lt, cl, cl, last, last, causal=True)
    loom.loom_attn_check_error()
    assert all(torch.equal(g[n:], w) for g, w in zip(got, want))


def test_a_skipped_copy_times_out_and_the_next_call_is_right(loom):
    loom.loom_attn_check_error()
    loom.loom_debug_set_timeout_ns(50_000_000)
    loom.loom_debug_inject(4)
    try:
        with pytest.raises(loom.LoomError) as e:
            _dense(loom, 1, 1, 1, 512, 512, 128, False, False)
        assert e.value.status == 6
    finally:
        loom.loom_debug_inject(0)
        loom.loom_debug_set_timeout_ns(0)
    host, grads = _dense(loom, 1, 1, 1, 512, 512, 128, False, False)
    _check_dense(host, grads, False, 128 ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("Hq,Hkv", [(16, 16), (8, 1)])
def test_a_skipped_copy_times_out_in_every_form(loom, Hq, Hkv, ragged, D):
    """Whole and split items (8 heads of one kv head)."""
    def call():
        if ragged:
            return _ragged(loom, (130, 900, 513), (130, 900, 513), Hq, Hkv, D, False, False)
        return _dense(loom, 1, Hq, Hkv, 700, 700, D, False, False)

    loom.loom_attn_check_error()
    loom.loom_debug_set_timeout_ns(50_000_000)
    loom.loom_debug_inject(4)
    try:
        with pytest.raises(loom.LoomError) as e:
            call()
        assert e.value.status == 6
    finally:
        loom.loom_debug_inject(0)
        loom.loom_debug_set_timeout_ns(0)
    out = call()
    if ragged:
        _check_ragged(*out, False, D ** -0.5)
    else:
        _check_dense(*out, False, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,kl", [((1, 900, 700), (1, 900, 700)), ((2, 5, 1200), (900, 1500, 1300)), ((40, 64), (2500, 1900))])
def test_few_long_ragged_items_are_split(loom, ql, kl, causal, D):
    """Few tiles with many steps, whose sums are split and joined (the workspace shows that they are);
    the same bits each time."""
    host, grads, cq, ck = _ragged(loom, ql, kl, 8, 1, D, causal, True)
    stats = 8 * (sum(ql) + 128 * len(ql)) * 8
    assert loom.loom_attn_bwd_varlen_workspace_bytes(len(ql), 8, 1, sum(ql), sum(kl), D) > 2 * stats
    _check_ragged(host, grads, cq, ck, causal, D ** -0.5)
    again = _ragged(loom, ql, kl, 8, 1, D, causal, True)[1]
    assert all((a == b).all() for a, b in zip(grads, again))


def test_refusals_of_the_binding(loom):
    import torch
    host, _ = _dense(loom, 1, 4, 2, 20, 20, 64, False, False)
    do, q, k, v, o, lse = [t.cuda() for t in host[:6]]
    with pytest.raises(TypeError):
        loom.loom_attn_bwd(do.float(), q, k, v, o, lse)
    with pytest.raises(TypeError):
        loom.loom_attn_bwd(do, q, k, v, o, lse.double())
    with pytest.raises(TypeError):
        loom.loom_attn_bwd(do, q, k, v, o, None)
    with pytest.raises(ValueError):
        loom.loom_attn_bwd(do, q.transpose(1, 2), k, v, o, lse)
    with pytest.raises(ValueError):
        loom.loom_attn_bwd(do[:, :2].contiguous(), q, k, v, o, lse)
    with pytest.raises(ValueError):
        loom.loom_attn_bwd(do, q, k, v, o, lse, dlse=lse[:, :2].contiguous())
    with pytest.raises(ValueError):
        loom.loom_attn_bwd(do, q, k, v, o, lse, dk=torch.empty_like(q))
    with pytest.raises(loom.LoomError) as e:
        loom.loom_attn_bwd(do, q, k, v, o, lse, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 4
    with pytest.raises(loom.LoomError) as e:
        loom.loom_attn_bwd(do, q, k, v, o, lse, scale=0.0)
    assert e.value.status == 1
