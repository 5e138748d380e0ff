"""Norm and rotation with positions on several axes, forward, into a cache and backward: against the formulas in
64 bits (tests/grad_ref.py), the angles taken pair by pair from each axis' row."""
import pytest

from tests import grad_ref as ref
from tests.test_gpu_qkv import SHAPES, Case, _within, loom  # noqa: F401

pytestmark = pytest.mark.gpu


class AxesCase(Case):
    def __init__(self, T, Hq, Hkv, D, R, S, interleaved=False, f32=False, axes=3, spread="turns", P=500, seed=0):
        import torch
        super().__init__(T, Hq, Hkv, D, R, S, interleaved, f32, extra=8 * (T % 3), P=P, seed=seed)
        half = R // 2
        self.axis = {"turns": [i % axes for i in range(half)], "blocks": [min(i * axes // half, axes - 1) for i in range(half)],
                     "last": [axes - 1] * half}[spread]
        self.pos = torch.randint(-3, P + 3, (axes, T), generator=self.gen).to(torch.int32)

    def heads(self):
        import torch
        x = self.rows[:, :(self.Hq + 2 * self.Hkv) * self.D].double().view(self.T, -1, self.D)
        row = self.pos.long().clamp(0, self.cos.shape[0] - 1)[self.axis].T  # [T, R / 2]
        pair = torch.arange(self.R // 2)
        return (x[:, :self.Hq], x[:, self.Hq:self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:], self.cos[row, pair].double(),
                self.sin[row, pair].double())


AXES = [(1, "last"), (2, "turns"), (3, "blocks"), (3, "turns"), (4, "turns"), (4, "last")]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes,spread", AXES)
@pytest.mark.parametrize("T,Hq,Hkv,D,R,S", SHAPES)
def test_forward(loom, T, Hq, Hkv, D, R, S, axes, spread, interleaved):  # noqa: F811
    c = AxesCase(T, Hq, Hkv, D, R, S, interleaved, T % 2 == 0, axes, spread)
    q, k, v = loom.loom_qkv_norm_rope(c.qkv, *c.args(), Hq, Hkv, c.pos.cuda(), seq_len=S, interleaved=interleaved, eps=c.eps,
                                      pair_axis=c.axis)
    (eq, bq), (ek, bk), ev = c.exact()
    assert q.shape == ((T // S, Hq, S, D) if S else (T, Hq, D))
    _within(c.tokens(q), eq, bq, "q")
    _within(c.tokens(k), ek, bk, "k")
    assert (c.tokens(v) == ev).all()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("axes,spread", AXES)
@pytest.mark.parametrize("T,Hq,Hkv,D,R,S", SHAPES)
def test_backward(loom, T, Hq, Hkv, D, R, S, axes, spread, interleaved):  # noqa: F811
    import torch
    c = AxesCase(T, Hq, Hkv, D, R, S, interleaved, T % 2 == 0, axes, spread, seed=1)
    shape = lambda H: (T // S, H, S, D) if S else (T, H, D)  # noqa: E731
    dq, dk, dv = (torch.randn(shape(h), generator=c.gen).bfloat16() for h in (Hq, Hkv, Hkv))
    dqkv, dqw, dkw = loom.loom_qkv_norm_rope_bwd(dq.cuda(), dk.cuda(), dv.cuda(), c.qkv, *c.args(), c.pos.cuda(),
                                                 interleaved=interleaved, eps=c.eps, pair_axis=tuple(c.axis))
    got = dqkv.double().cpu().view(T, -1, D)
    xq, xk, _, co, si = c.heads()
    for dy, x, w, dw, at, n in ((dq, xq, c.qw, dqw, 0, "q"), (dk, xk, c.kw, dkw, Hq, "k")):
        (dx, dwe), (bx, bw) = ref.norm_rope_grads(c.tokens(dy), x, w.double(), co, si, R, interleaved, c.eps)
        _within(got[:, at:at + x.shape[1]], dx, bx, f"dqkv's {n} heads")
        _within(dw.double().cpu(), dwe, bw, f"d{n}_weight")
    assert (got[:, Hq + Hkv:] == c.tokens(dv)).all()


@pytest.mark.parametrize("layout", ["nhd", "hnd"])
@pytest.mark.parametrize("T,Hq,Hkv,D,R,page", [(1, 32, 8, 128, 128, 16), (70, 6, 3, 64, 48, 5), (300, 28, 4, 128, 128, 64)])
def test_into_a_cache(loom, T, Hq, Hkv, D, R, page, layout):  # noqa: F811
    import torch
    c = AxesCase(T, Hq, Hkv, D, R, 0)
    pages = T // page + 3
    k, v = (torch.full((pages, page, Hkv, D) if layout == "nhd" else (pages, Hkv, page, D), 9.0, dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    slots = torch.randperm(pages * page, generator=c.gen)[:T].to(torch.int32)
    slots[T // 2] = -1
    q = loom.loom_qkv_norm_rope_cache(c.qkv, *c.args(), c.pos.cuda(), slots.cuda(), k, v, Hq, layout=layout, eps=c.eps,
                                      pair_axis=c.axis)
    (eq, bq), (ek, bk), ev = c.exact()
    _within(q.double().cpu(), eq, bq, "q")
    k, v = ((x if layout == "nhd" else x.transpose(1, 2)).double().cpu().reshape(-1, Hkv, D) for x in (k, v))
    w = slots >= 0
    _within(k[slots[w].long()], ek[w], bk[w], "k")
    assert (v[slots[w].long()] == ev[w]).all()
    rest = torch.ones(len(k), dtype=torch.bool)
    rest[slots[w].long()] = False
    assert (k[rest] == 9).all() and (v[rest] == 9).all()


def test_one_axis_is_the_call_without(loom):  # noqa: F811
    """All axes alike, and one axis alone, give the call without axes to the bit."""
    import torch
    c = AxesCase(300, 8, 2, 128, 96, 0)
    pos = c.pos[0].cuda()
    for inter in (False, True):
        want = loom.loom_qkv_norm_rope(c.qkv, *c.args(), 8, 2, pos, interleaved=inter)
        for p, axis in ((pos[None], [0] * 48), (pos.expand(3, -1).contiguous(), c.axis)):
            got = loom.loom_qkv_norm_rope(c.qkv, *c.args(), 8, 2, p, interleaved=inter, pair_axis=axis)
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        grads = [torch.randn(x.shape, device="cuda").bfloat16() for x in want]
        want = loom.loom_qkv_norm_rope_bwd(*grads, c.qkv, *c.args(), pos, interleaved=inter)
        got = loom.loom_qkv_norm_rope_bwd(*grads, c.qkv, *c.args(), pos.expand(3, -1).contiguous(), interleaved=inter, pair_axis=c.axis)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_gradients_through_autograd(loom):  # noqa: F811
    """The gradient of a weighted sum of q, k and v against differences of it, in 64 bits by the formula."""
    import torch
    from paper_2609_29219_gb300 import autograd
    c = AxesCase(40, 3, 2, 64, 64, 0, seed=2)
    w = [torch.randn((40, h, 64), generator=c.gen).bfloat16() for h in (3, 2, 2)]
    x = c.qkv.detach().contiguous().requires_grad_()
    qw, kw, cos, sin = c.args()
    out = autograd.qkv_norm_rope(x, qw, kw, cos, sin, 3, 2, c.pos.cuda(), eps=c.eps, pair_axis=c.axis)
    sum((o * g.cuda()).float().sum() for o, g in zip(out, w)).backward()
    xq, xk, xv, co, si = c.heads()
    full = torch.cat((xq, xk, xv), 1)

    def loss(x):
        q = ref.norm_rope(x[:, :3], c.qw.double(), co, si, 64, False, c.eps)
        k = ref.norm_rope(x[:, 3:5], c.kw.double(), co, si, 64, False, c.eps)
        return sum((a * b.double()).sum() for a, b in zip((q, k, x[:, 5:]), w))

    (dq, _), (bq, _) = ref.norm_rope_grads(w[0].double(), xq, c.qw.double(), co, si, 64, False, c.eps)
    (dk, _), (bk, _) = ref.norm_rope_grads(w[1].double(), xk, c.kw.double(), co, si, 64, False, c.eps)
    got = x.grad.double().cpu().view(40, -1, 64)
    bound = torch.cat((bq, bk, torch.zeros_like(xv)), 1)
    for seed in range(4):
        d = torch.randn(full.shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * full.abs().clamp(min=1e-3)
        h = 1e-5
        change = (loss(full + h * d) - loss(full - h * d)) / (2 * h)
        assert abs((got * d).sum() - change) <= (bound * d.abs()).sum() + 1e-6 * abs(change) + 1e-6


def test_axes_in_a_list_that_changes(loom):  # noqa: F811
    """What pair_axis was is read at the call: a list or a tensor's numbers changed since are other axes."""
    import torch
    c = AxesCase(10, 4, 2, 64, 32, 0)
    call = lambda axis: loom.loom_qkv_norm_rope(c.qkv, *c.args(), 4, 2, c.pos.cuda(), pair_axis=axis)[0]  # noqa: E731
    one, other = [0] * 16, [1] * 16
    for kind in (list, torch.tensor, lambda x: tuple(torch.tensor(x))):
        axis = kind(one)
        assert torch.equal(call(axis), call(tuple(one)))
        for i in range(16):
            axis[i].fill_(1) if isinstance(axis, tuple) else axis.__setitem__(i, 1)
        assert torch.equal(call(axis), call(tuple(other))) and not torch.equal(call(axis), call(tuple(one)))


def test_refusals(loom):  # noqa: F811
    c = AxesCase(10, 4, 2, 64, 32, 0)
    call = lambda pos, axis, **kw: loom.loom_qkv_norm_rope(c.qkv, *c.args(), 4, 2, pos, pair_axis=axis, **kw)  # noqa: E731
    pos = c.pos.cuda()
    with pytest.raises(TypeError, match="positions are needed"):
        call(None, c.axis)
    with pytest.raises(ValueError, match="2 dims"):
        call(pos[0], c.axis)
    with pytest.raises(ValueError, match="contiguous"):
        call(pos.T.contiguous().T, c.axis)
    with pytest.raises(TypeError, match="int32"):
        call(pos.long(), c.axis)
    with pytest.raises(ValueError, match=r"\[axes, T\]"):
        call(pos[:, :9].contiguous(), c.axis)
    with pytest.raises(ValueError, match="16 pairs"):
        call(pos, c.axis[:-1])
    with pytest.raises(ValueError, match="does not|do not have"):
        call(pos, [3] * 16)
    with pytest.raises(ValueError, match="do not have"):
        call(pos, [-1] * 16)
    with pytest.raises(TypeError, match="integer"):
        call(pos, [0.5] * 16)
    with pytest.raises(loom.LoomError, match="UNSUPPORTED"):
        call(pos[:1].expand(5, -1).contiguous(), c.axis)
    with pytest.raises(ValueError, match="1 dims"):
        loom.loom_qkv_norm_rope(c.qkv, *c.args(), 4, 2, pos)
