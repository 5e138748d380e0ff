"""Argument checks of the chunk's attention, the step's bookkeeping and positions on several axes, none of
which needs a GPU."""
import ctypes

import pytest

FAKE = 0x10000  # aligned, never dereferenced: every call below is rejected during validation
HUGE = (1 << 31) - 1


@pytest.fixture(scope="module")
def lib():
    from paper_2609_29219_gb300 import build
    build.build()
    import paper_2609_29219_gb300 as loom
    return loom.capi()


def _caller(fn, ok):
    def call(**kw):
        a = dict(ok)
        assert set(kw) <= set(a)
        a.update(kw)
        return fn(*a.values())
    return call


CHUNK = dict(q=FAKE, k=FAKE, v=FAKE, table=FAKE, cu=FAKE, lens=FAKE, o=FAKE, lse=None, ws=FAKE, wsb=1 << 30, B=2, Hq=8, Hkv=2,
             T=100, pages=50, page=16, most=10, layout=0, D=64, causal=1, scale=0.125, stream=None)


@pytest.mark.parametrize("change,expect", [
    ({"q": None}, 1), ({"k": None}, 1), ({"table": None}, 1), ({"cu": None}, 1), ({"lens": None}, 1), ({"o": None}, 1),
    ({"B": 0}, 1), ({"Hq": 7}, 1), ({"Hkv": 0}, 1), ({"T": -1}, 1), ({"pages": 0}, 1), ({"page": 0}, 1), ({"most": 0}, 1),
    ({"layout": 2}, 1), ({"causal": 2}, 1), ({"scale": 0.0}, 1), ({"scale": float("nan")}, 1), ({"scale": float("inf")}, 1),
    ({"D": 96}, 2), ({"page": 24}, 2), ({"page": 4}, 2), ({"page": 65}, 2), ({"pages": HUGE}, 2), ({"most": HUGE}, 2),
    ({"T": HUGE}, 2), ({"T": 1, "Hq": 1 << 17}, 2), ({"q": FAKE + 8}, 3), ({"v": FAKE + 2}, 3), ({"o": FAKE + 4}, 3), ({"lse": FAKE + 2}, 3),
    ({"table": FAKE + 1}, 3), ({"cu": FAKE + 2}, 3), ({"lens": FAKE + 2}, 3), ({"ws": None}, 4), ({"wsb": 100}, 4),
    ({"ws": FAKE + 8}, 3)])
def test_chunk_rejects(lib, change, expect):
    assert _caller(lib.loom_attn_chunk_paged, CHUNK)(**change) == expect


def test_chunk_without_tokens(lib):
    assert _caller(lib.loom_attn_chunk_paged, CHUNK)(T=0, q=None, o=None, ws=None) == 0


def test_chunk_workspace(lib):
    need = lib.loom_attn_chunk_paged_workspace_bytes
    assert 0 < need(1, 32, 8, 1, 128) <= need(64, 32, 8, 5000, 128) <= 41 << 20
    assert need(1, 32, 5, 1, 128) == 0 and need(0, 32, 8, 1, 128) == 0 and need(1, 32, 8, 1, 96) == 0
    assert need(1, 32, 8, -1, 128) == 0 and need(1, 32, 8, HUGE, 128) == 0


PLAN = dict(new=FAKE, lens=FAKE, table=FAKE, free=FAKE, count=FAKE, count_out=FAKE, cu=FAKE, seqlens=FAKE, pos=FAKE, slots=FAKE,
            granted=FAKE, B=4, T=10, pages=50, page=16, most=10, stream=None)


@pytest.mark.parametrize("change,expect", [({n: None}, 1) for n in list(PLAN)[:11]] + [
    ({n: FAKE + 2}, 3) for n in list(PLAN)[:11]] + [
    ({"B": 0}, 1), ({"T": -1}, 1), ({"pages": 0}, 1), ({"page": 0}, 1), ({"most": 0}, 1), ({"B": 8193}, 2),
    ({"pages": HUGE}, 2), ({"most": HUGE}, 2), ({"page": HUGE}, 2)])
def test_plan_rejects(lib, change, expect):
    assert _caller(lib.loom_paged_plan, PLAN)(**change) == expect


AXIS = (ctypes.c_int * 32)(*(i % 3 for i in range(32)))
BAD_AXIS = (ctypes.c_int * 32)(*([0] * 31 + [3]))
LOW_AXIS = (ctypes.c_int * 32)(*([0] * 31 + [-1]))
NORM = dict(qkv=FAKE, stride=12 * 64, qw=FAKE, kw=FAKE, wt=0, cos=FAKE, sin=FAKE, P=100, R=64, inter=0, pos=FAKE, pstride=6, axes=3,
            axis=AXIS)
SIZES = dict(T=6, S=3, Hq=8, Hkv=2, D=64, eps=1e-6, stream=None)
FWD = dict(NORM, q=FAKE, k=FAKE, v=FAKE, **SIZES)
CACHE = dict(NORM, slots=FAKE, q=FAKE, kc=FAKE, vc=FAKE, pages=10, page=16, layout=0, T=6, Hq=8, Hkv=2, D=64, eps=1e-6, stream=None)
NBWD = dict(dq=FAKE, dk=FAKE, dv=FAKE, **NORM, dqkv=FAKE, dstride=12 * 64, dqw=FAKE, dkw=FAKE, ws=FAKE, wsb=1 << 30, **SIZES)
CALLS = [("loom_qkv_norm_rope_axes", FWD), ("loom_qkv_norm_rope_axes_cache", CACHE), ("loom_qkv_norm_rope_axes_bwd", NBWD)]


@pytest.mark.parametrize("name,ok", CALLS)
@pytest.mark.parametrize("change,expect", [
    ({"pos": None}, 1), ({"pstride": 5}, 1), ({"axes": 0}, 1), ({"axes": 5}, 2), ({"axis": None}, 1), ({"axis": BAD_AXIS}, 1),
    ({"axis": LOW_AXIS}, 1), ({"axes": 2}, 1), ({"qkv": None}, 1), ({"R": 24}, 2), ({"D": 96}, 2), ({"pos": FAKE + 2}, 3),
    ({"cos": FAKE + 4}, 3), ({"eps": 0.0}, 1), ({"T": -1}, 1)])
def test_axes_reject(lib, name, ok, change, expect):
    assert _caller(getattr(lib, name), ok)(**change) == expect


def test_axes_nothing_to_do(lib):
    assert _caller(lib.loom_qkv_norm_rope_axes, FWD)(T=0, S=0) == 0
    assert _caller(lib.loom_qkv_norm_rope_axes_cache, CACHE)(T=0, pos=None) == 0
