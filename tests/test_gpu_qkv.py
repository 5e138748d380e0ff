"""Norms of q and k per head with the rotation, forward, into a cache and backward, against the
formulas in 64 bits (tests/grad_ref.py)."""
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


class Case:
    def __init__(self, T, Hq, Hkv, D, R, seq_len=0, interleaved=False, f32=False, extra=0, P=500, seed=0, eps=1e-6):
        import torch
        gen = torch.Generator().manual_seed(seed)
        self.T, self.Hq, self.Hkv, self.D, self.R, self.S = T, Hq, Hkv, D, R, seq_len
        self.interleaved, self.eps = interleaved, eps
        W = (Hq + 2 * Hkv) * D
        rows = torch.randn((T, W + extra), generator=gen) * torch.exp(2 * torch.randn((T, 1), generator=gen))
        self.rows = rows.bfloat16()
        self.qw, self.kw = ((1 + 0.3 * torch.randn(D, generator=gen)).to(torch.float32 if f32 else torch.bfloat16) for _ in range(2))
        angle = torch.arange(P)[:, None] * 100.0 ** (-torch.arange(R // 2) / (R // 2))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.pos = None if seq_len else torch.randint(0, P, (T,), generator=gen).to(torch.int32)
        self.dev_rows = self.rows.cuda()
        self.qkv = self.dev_rows[:, :W]
        self.gen = gen

    def args(self):
        return self.qw.cuda(), self.kw.cuda(), self.cos.cuda(), self.sin.cuda()

    def heads(self):
        import torch
        x = self.rows[:, :(self.Hq + 2 * self.Hkv) * self.D].double().view(self.T, -1, self.D)
        pos = (torch.arange(self.T) % self.S if self.S else self.pos.long()).clamp(0, self.cos.shape[0] - 1)
        return (x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:], self.cos[pos].double(),
                self.sin[pos].double())

    def exact(self):
        """(q, k) in 64 bits with bounds: rounded once to bf16, the rest fp32; and v as it is."""
        xq, xk, xv, c, s = self.heads()
        out = []
        for x, w in ((xq, self.qw), (xk, self.kw)):
            w = w.double()
            y = ref.norm_rope(x, w, c, s, self.R, self.interleaved, self.eps)
            a = (x * w).abs() / ((x * x).mean(-1, keepdim=True) + self.eps).sqrt()
            mag = ref.rotate(a, c.abs(), s.abs(), self.R, self.interleaved).abs().maximum(
                ref.rotate(a, c.abs(), -s.abs(), self.R, self.interleaved).abs())
            out.append((y, 1.01 * ref.BF16 * y.abs() + ref.FP32 * mag + 1e-30))
        return out[0], out[1], xv

    def tokens(self, t):
        """[T, H, D] of an output or gradient laid out for attention."""
        t = t.double().cpu()
        return t.transpose(1, 2).reshape(self.T, t.shape[1], self.D) if self.S else t


def _within(got, exact, bound, what):
    import torch
    assert got.shape == exact.shape and torch.isfinite(got).all(), what
    over = (got - exact).abs() - bound
    assert not (over > 0).any(), f"{what}: {int((over > 0).sum())} of {over.numel()} past the bound, worst {float(over.max()):.3g}"


SHAPES = [  # T, Hq, Hkv, D, R, seq_len
    (1, 1, 1, 64, 64, 0), (1, 32, 8, 128, 128, 0), (7, 6, 3, 128, 64, 0), (60, 8, 1, 64, 48, 20), (33, 5, 5, 128, 16, 0),
    (300, 16, 2, 64, 16, 100), (1000, 3, 1, 128, 112, 1), (257, 32, 32, 64, 64, 0)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,R,S", SHAPES)
def test_forward(loom, T, Hq, Hkv, D, R, S, f32, interleaved):
    c = Case(T, Hq, Hkv, D, R, S, interleaved, f32, extra=8 * (T % 3))
    q, k, v = loom.loom_qkv_norm_rope(c.qkv, *c.args(), Hq, Hkv, None if c.pos is None else c.pos.cuda(), seq_len=S,
                                      interleaved=interleaved, eps=c.eps)
    (eq, bq), (ek, bk), ev = c.exact()
    assert q.shape == ((T // S, Hq, S, D) if S else (T, Hq, D)) and q.is_contiguous() and v.is_contiguous()
    _within(c.tokens(q), eq, bq, "q")
    _within(c.tokens(k), ek, bk, "k")
    assert (c.tokens(v) == ev).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D,R,S", SHAPES)
def test_backward(loom, T, Hq, Hkv, D, R, S, f32, interleaved):
    import torch
    c = Case(T, Hq, Hkv, D, R, S, interleaved, f32, extra=8 * (T % 3), seed=1)
    shape = lambda H: (T // S, H, S, D) if S else (T, H, D)  # noqa: E731
    dq, dk, dv = (torch.randn(shape(h), generator=c.gen).bfloat16() for h in (Hq, Hkv, Hkv))
    dqkv, dqw, dkw = loom.loom_qkv_norm_rope_bwd(dq.cuda(), dk.cuda(), dv.cuda(), c.qkv, *c.args(),
                                                 None if c.pos is None else c.pos.cuda(), interleaved=interleaved, eps=c.eps)
    got = dqkv.double().cpu().view(T, -1, D)
    xq, xk, _, co, si = c.heads()
    for dy, x, w, dw, at, n in ((dq, xq, c.qw, dqw, 0, "q"), (dk, xk, c.kw, dkw, Hq, "k")):
        (dx, dwe), (bx, bw) = ref.norm_rope_grads(c.tokens(dy), x, w.double(), co, si, R, interleaved, c.eps)
        _within(got[:, at:at + x.shape[1]], dx, bx, f"dqkv's {n} heads")
        _within(dw.double().cpu(), dwe, bw, f"d{n}_weight")
    assert (got[:, Hq + Hkv:] == c.tokens(dv)).all()


def test_gradient_against_differences_of_the_loss(loom):
    import torch
    c = Case(40, 3, 2, 64, 64, 0, seed=2)
    dq, dk, dv = (torch.randn((40, h, 64), generator=c.gen).bfloat16() for h in (3, 2, 2))
    got = loom.loom_qkv_norm_rope_bwd(dq.cuda(), dk.cuda(), dv.cuda(), c.qkv, *c.args(), c.pos.cuda(), eps=c.eps)
    xq, xk, xv, co, si = c.heads()
    x = torch.cat((xq, xk, xv), 1)

    def loss(x, qw, kw):
        f = lambda y, w: ref.norm_rope(y, w, co, si, 64, False, c.eps)  # noqa: E731
        return (f(x[:, :3], qw) * dq).sum() + (f(x[:, 3:5], kw) * dk).sum() + (x[:, 5:] * dv).sum()

    at = (x, c.qw.double(), c.kw.double())
    for i in range(3):
        # a step in proportion to the values: a token's heads go from 1e-2 to 1e2
        u = torch.randn(at[i].shape, generator=c.gen, dtype=torch.float64) * at[i].abs()
        h = 1e-5
        slope = (loss(*[y + h * u if j == i else y for j, y in enumerate(at)])
                 - loss(*[y - h * u if j == i else y for j, y in enumerate(at)])) / (2 * h)
        g = got[i].double().cpu().view(at[i].shape)
        # one rounding to bf16, fp32 for the rest; dx is a difference of terms up to ten times itself
        assert abs((g * u).sum() - slope) <= (ref.BF16 + 10 * ref.FP32) * (g * u).abs().sum() + 1e-6


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("T,Hq,Hkv,D,R,page", [(1, 32, 8, 128, 128, 16), (5, 4, 2, 64, 32, 1), (100, 6, 3, 128, 128, 48),
                                               (260, 8, 1, 64, 64, 5)])
def test_cache_form(loom, T, Hq, Hkv, D, R, page, layout):
    import torch
    c = Case(T, Hq, Hkv, D, R, extra=8, seed=3)
    pages = T // page + 3
    shape = (pages, page, Hkv, D) if layout == "nhd" else (pages, Hkv, page, D)
    before = [torch.randn(shape, generator=c.gen).bfloat16() for _ in range(2)]
    kc, vc = [t.cuda() for t in before]
    slots = torch.randperm(pages * page, generator=c.gen)[:T].to(torch.int32)
    if T > 4:  # padding: below and past the cache
        slots[1], slots[3] = -1, pages * page
    q = loom.loom_qkv_norm_rope_cache(c.qkv, *c.args(), c.pos.cuda(), slots.cuda(), kc, vc, Hq, layout=layout)
    (eq, bq), (ek, bk), ev = c.exact()
    _within(q.double().cpu(), eq, bq, "q")
    rows = lambda t: t.cpu().double() if layout == "nhd" else t.cpu().double().transpose(1, 2)  # noqa: E731
    fk, fv, ok, ov = [rows(t).reshape(pages * page, Hkv, D).clone() for t in (kc, vc, *before)]
    keep = (slots >= 0) & (slots < pages * page)
    at = slots[keep].long()
    _within(fk[at], ek[keep], bk[keep], "k_cache")
    assert (fv[at] == ev[keep]).all()
    fk[at], fv[at] = ok[at], ov[at]
    assert (fk == ok).all() and (fv == ov).all()  # nothing else was written


def test_cache_offsets_past_32_bits(loom):
    """A contiguous cache [B, Hkv, capacity, D] of more than 2^31 values: rows at its far end."""
    import torch
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    B, Hq, Hkv, cap, D = 3, 8, 4, 1_500_000, 128
    c = Case(B, Hq, Hkv, D, 128, seed=4)
    kc, vc = (torch.zeros((B, Hkv, cap, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    where = [cap - 1, 0, cap - 2]
    slots = torch.tensor([b * cap + p for b, p in enumerate(where)], dtype=torch.int32, device="cuda")
    loom.loom_qkv_norm_rope_cache(c.qkv, *c.args(), c.pos.cuda(), slots, kc, vc, Hq, layout="hnd")
    _, (ek, bk), ev = c.exact()
    for b, p in enumerate(where):
        _within(kc[b, :, p].double().cpu(), ek[b], bk[b], "k")
        assert (vc[b, :, p].double().cpu() == ev[b]).all()
        vc[b, :, p] = 0
    assert not vc.any()


def test_positions_are_clamped_to_the_tables(loom):
    import torch
    c = Case(4, 2, 1, 64, 64, P=10)
    c.pos = torch.tensor([-5, 0, 9, 1 << 30], dtype=torch.int32)
    q, _, _ = loom.loom_qkv_norm_rope(c.qkv, *c.args(), 2, 1, c.pos.cuda())
    (eq, bq), _, _ = c.exact()
    _within(c.tokens(q), eq, bq, "q")


def test_rows_between_are_left_alone_and_empty_calls(loom):
    import torch
    c = Case(20, 2, 1, 64, 32, extra=16)
    dq, dk = torch.ones((20, 2, 64), device="cuda").bfloat16(), torch.ones((20, 1, 64), device="cuda").bfloat16()
    into = torch.full((20, 256 + 24), 7.0, device="cuda").bfloat16()
    out, dqw, dkw = loom.loom_qkv_norm_rope_bwd(dq, dk, dk, c.qkv, *c.args(), c.pos.cuda(), dqkv=into[:, :256])
    plain, a, b = loom.loom_qkv_norm_rope_bwd(dq, dk, dk, c.qkv, *c.args(), c.pos.cuda())
    assert torch.equal(out, plain) and torch.equal(dqw, a) and torch.equal(dkw, b) and (into[:, 256:] == 7).all()
    none = c.qkv[:0].contiguous()
    q, k, v = loom.loom_qkv_norm_rope(none, *c.args(), 2, 1)
    assert q.shape == (0, 2, 64) and v.shape == (0, 1, 64)
    dqw, dkw = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
    loom.loom_qkv_norm_rope_bwd(dq[:0], dk[:0], dk[:0], none, *c.args(), dq_weight=dqw, dk_weight=dkw)
    assert not dqw.any() and not dkw.any()


@pytest.mark.parametrize("T,Hq,Hkv,D", [(2, 2433, 3, 128), (9, 2433, 3, 128), (1, 16382, 1, 64), (2, 9000, 1, 128)])
def test_heads_that_do_not_divide_the_warps(loom, T, Hq, Hkv, D):
    """A token's units (307 of the first two, prime) are no divisor of the grid's warps."""
    test_forward(loom, T, Hq, Hkv, D, 32, 0, True, False)
    test_backward(loom, T, Hq, Hkv, D, 32, 0, True, False)


def test_the_same_inputs_give_the_same_bits_on_any_stream(loom):
    import torch
    c = Case(5000, 16, 4, 64, 64, seed=5)
    dq, dk, dv = (torch.randn((5000, h, 64), generator=c.gen).bfloat16().cuda() for h in (16, 4, 4))
    args = (dq, dk, dv, c.qkv, *c.args(), c.pos.cuda())
    a = loom.loom_qkv_norm_rope_bwd(*args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ws = torch.full((loom.loom_qkv_norm_rope_bwd_workspace_bytes(64),), 255, dtype=torch.uint8, device="cuda")
        b = loom.loom_qkv_norm_rope_bwd(*args, workspace=ws)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refusals_of_the_binding(loom):
    import torch
    c = Case(6, 2, 1, 64, 32)
    qw, kw, cos, sin = c.args()
    with pytest.raises(TypeError):
        loom.loom_qkv_norm_rope(c.qkv.float(), qw, kw, cos, sin, 2, 1)
    with pytest.raises(TypeError):
        loom.loom_qkv_norm_rope(c.qkv, qw, kw.float(), cos, sin, 2, 1)
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope(c.qkv, qw, kw, cos, sin, 3, 1)
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope(c.qkv, qw, kw, cos, sin, 2, 1, seq_len=4)
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope(c.qkv, qw, kw, cos, sin[:5].contiguous(), 2, 1)
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope(c.qkv.t().contiguous().t(), qw, kw, cos, sin, 2, 1)
    with pytest.raises(loom.LoomError) as e:
        loom.loom_qkv_norm_rope(c.qkv, qw, kw, cos[:, :4].contiguous(), sin[:, :4].contiguous(), 2, 1)
    assert e.value.status == 2
    with pytest.raises(loom.LoomError) as e:
        loom.loom_qkv_norm_rope(c.qkv, qw, kw, cos, sin, 2, 1, eps=0.0)
    assert e.value.status == 1
    cache = torch.zeros((2, 16, 1, 64), device="cuda").bfloat16()
    with pytest.raises(TypeError):
        loom.loom_qkv_norm_rope_cache(c.qkv, qw, kw, cos, sin, None, None, cache, cache, 2)
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope_cache(c.qkv, qw, kw, cos, sin, c.pos.cuda(), c.pos.cuda()[:3].contiguous(), cache, cache, 2)
    dq = torch.zeros((6, 2, 64), device="cuda").bfloat16()
    with pytest.raises(ValueError):
        loom.loom_qkv_norm_rope_bwd(dq, dq, dq, c.qkv, qw, kw, cos, sin)
