"""The backward pass in each way that its work is dealt, against the formulas in 64 bits: CTAs that take
several whole items of keys, split items of keys, of query rows and of both, dense and ragged."""
import pytest

from tests.test_gpu_bwd import _check_dense, _check_ragged, _dense, _ragged, loom  # noqa: F401

pytestmark = pytest.mark.gpu


def _shares(loom, *sizes, **kw):  # noqa: F811
    plan = loom.loom_attn_bwd_plan(*sizes, **kw)
    return plan["kv_shares"], plan["q_shares"]


def _sms():
    import torch
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv", [(2, 32, 32, 700, 700), (4, 24, 12, 515, 601), (5, 30, 10, 400, 500), (7, 16, 16, 129, 300)])
def test_ctas_take_several_whole_items(loom, B, Hq, Hkv, Sq, Skv, D, causal):  # noqa: F811
    import torch
    assert _shares(loom, B, Hq, Hkv, Sq, Skv, D, causal) == (1, 1)
    assert B * Hkv * -(-Skv // 128) > _sms()
    host, grads = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, dlse=Hq > Hkv)
    _check_dense(host, grads, causal, D ** -0.5)
    again = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, dlse=Hq > Hkv)[1]
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,Skv,kv,q", [(1, 8, 1, 700, 700, True, False), (1, 2, 1, 300, 4000, False, True),
                                                  (1, 4, 1, 1000, 4000, True, True)])
def test_split_items(loom, B, Hq, Hkv, Sq, Skv, kv, q, D, causal):  # noqa: F811
    import torch
    shares = _shares(loom, B, Hq, Hkv, Sq, Skv, D, causal)
    assert (shares[0] > 1, shares[1] > 1) == (kv, q)
    host, grads = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, True)
    _check_dense(host, grads, causal, D ** -0.5)
    again = _dense(loom, B, Hq, Hkv, Sq, Skv, D, causal, True)[1]
    assert all(torch.equal(x, y) for x, y in zip(grads, again))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ql,kl,H,kv,q", [
    ((1, 900, 700), (1, 900, 700), (8, 1), True, False),       # shares without steps
    ((2, 5, 1200), (900, 1500, 3), (8, 1), True, False),       # ... and, causal, rows that see nothing
    ((0, 1000, 300), (700, 0, 40), (8, 1), True, False),       # sequences without queries, without keys
    ((64, 100, 30), (3000, 2500, 10), (4, 4), False, True),    # rows that see nothing
    ((1000,), (4000,), (4, 1), True, True),
    ((1000,), (4000,), (3, 1), True, True),
])
def test_split_ragged_items(loom, ql, kl, H, kv, q, D, causal):  # noqa: F811
    shares = _shares(loom, len(ql), *H, sum(ql), sum(kl), D, causal, True)
    assert (shares[0] > 1, shares[1] > 1) == (kv, q)
    host, grads, cq, ck = _ragged(loom, ql, kl, *H, D, causal, True)
    _check_ragged(host, grads, cq, ck, causal, D ** -0.5)
    again = _ragged(loom, ql, kl, *H, D, causal, True)[1]
    assert all((a == b).all() for a, b in zip(grads, again))
