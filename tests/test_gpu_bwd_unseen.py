"""Rows that see nothing (a causal sequence of more queries than keys): whatever they and their
gradients hold reaches no gradient, and their own is zero."""
import pytest

from tests import grad_ref as ref
from tests.test_gpu_bwd import _check_ragged, loom  # noqa: F401

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _case(ql, kl, Hq, Hkv, D, seed=0):
    """Inputs on the host whose unseen rows hold zeros, LSE of -inf among them; and where those rows are."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    mk = lambda n, h: torch.randn((n, h, D), generator=gen).bfloat16()  # noqa: E731
    q, k, v, do = mk(sum(ql), Hq), mk(sum(kl), Hkv), mk(sum(kl), Hkv), mk(sum(ql), Hq)
    dl = torch.randn((Hq, sum(ql)), generator=gen)
    cq, ck = [torch.tensor([0] + list(x)).cumsum(0).to(torch.int32) for x in (ql, kl)]
    o, lse = torch.zeros(sum(ql), Hq, D), torch.full((Hq, sum(ql)), -INF)
    unseen = torch.zeros(sum(ql), dtype=torch.bool)
    for b, (n, m) in enumerate(zip(ql, kl)):
        a, c = int(cq[b]), int(ck[b])
        unseen[a:a + max(0, n - m)] = True
        if n and m:
            x, y = ref.attention(q[a:a + n].transpose(0, 1).double(), k[c:c + m].transpose(0, 1).double(),
                                 v[c:c + m].transpose(0, 1).double(), True, D ** -0.5)
            o[a:a + n], lse[:, a:a + n] = x.transpose(0, 1).float(), y.float()
    q[unseen], do[unseen], dl[:, unseen] = 0, 0, 0
    return [do, q, k, v, o.bfloat16(), lse, dl], cq, ck, unseen


# sq - skv no multiple of a tile, of a tile and within one, with sequences on both sides
LENGTHS = [((5, 200, 130), (260, 40, 130)), ((300, 64), (40, 64)), ((257, 129, 30), (1, 128, 30)), ((40, 1200, 9), (70, 900, 9))]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(6, 3), (8, 1)])
@pytest.mark.parametrize("ql,kl", LENGTHS)
@pytest.mark.parametrize("what", ["dlse -inf", "dlse nan", "o", "do", "q", "all"])
def test_what_unseen_rows_hold_reaches_nothing(loom, what, ql, kl, Hq, Hkv, D):  # noqa: F811
    host, cq, ck, unseen = _case(ql, kl, Hq, Hkv, D)
    given = [t.clone() for t in host]
    if what in ("dlse -inf", "dlse nan", "all"):
        given[6][:, unseen] = -INF if what == "dlse -inf" else NAN
    if what in ("o", "all"):
        given[4][unseen] = NAN
    if what in ("do", "all"):
        given[0][unseen] = INF
    if what in ("q", "all"):
        given[1][unseen] = NAN
    do, q, k, v, o, lse, dl = [t.cuda() for t in given]
    grads = loom.loom_attn_bwd_varlen(do, q, k, v, o, lse, cq.cuda(), ck.cuda(), max(ql), max(kl), causal=True, dlse=dl)
    loom.loom_attn_check_error()
    assert (grads[0][unseen] == 0).all()
    _check_ragged(host, grads, cq.tolist(), ck.tolist(), True, D ** -0.5)


def test_a_row_without_probability_ignores_its_statistics(loom):  # noqa: F811
    """Dense: LSE of -inf given for a row, its gradient of LSE -inf."""
    import torch
    gen = torch.Generator().manual_seed(1)
    mk = lambda h: torch.randn((1, h, 140, 64), generator=gen).bfloat16()  # noqa: E731
    do, q, k, v = mk(4), mk(4), mk(2), mk(2)
    o, lse = ref.attention(q[0].double(), k[0].double(), v[0].double(), False, 0.125)
    o, lse, dl = o[None].bfloat16(), lse[None].float(), torch.zeros((1, 4, 140))
    lse[..., 7], dl[..., 7] = -INF, -INF
    got = loom.loom_attn_bwd(*[t.cuda() for t in (do, q, k, v, o, lse)], dlse=dl.cuda())
    loom.loom_attn_check_error()
    assert (got[0][:, :, 7] == 0).all()
    rows = torch.arange(140) != 7  # the others' gradients are those of a call without the row
    kept = [t[0].double()[:, rows] for t in (do, q)] + [k[0].double(), v[0].double()] + [t[0].double()[:, rows] for t in (o, lse)]
    exact, bound = ref.attention_grads(*kept, None, False, 0.125)
    for g, e, b, at in zip(got, exact, bound, (rows, slice(None), slice(None))):
        g = g[0].double().cpu()[:, at]
        assert torch.isfinite(g).all() and ((g - e).abs() <= b).all()
