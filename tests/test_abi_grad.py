"""Argument checks of the training and serving entry points, none of which needs a GPU."""
import pytest

FAKE = 0x10000  # aligned, never dereferenced: every call below is rejected during validation


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


BWD = dict(do=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dlse=None, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, wsb=1 << 30, B=2,
           Hq=8, Hkv=2, Sq=100, Skv=120, D=64, causal=1, scale=0.125, stream=None)


@pytest.mark.parametrize("change,expect", [
    ({"do": None}, 1), ({"lse": None}, 1), ({"dv": None}, 1), ({"B": 0}, 1), ({"Sq": 0}, 1), ({"Hq": 7}, 1),
    ({"causal": 2}, 1), ({"Sq": 121}, 1), ({"scale": 0.0}, 1), ({"scale": float("inf")}, 1), ({"D": 96}, 2),
    ({"B": 1 << 20, "Sq": 1 << 20, "Skv": 1 << 20}, 2), ({"q": FAKE + 8}, 3), ({"dk": FAKE + 2}, 3), ({"lse": FAKE + 2}, 3),
    ({"dlse": FAKE + 1}, 3), ({"ws": None}, 4), ({"wsb": 100}, 4), ({"ws": FAKE + 8}, 3)])
def test_attn_bwd_rejects(lib, change, expect):
    assert _caller(lib.loom_attn_bwd, BWD)(**change) == expect


VAR = dict(do=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, dlse=None, dq=FAKE, dk=FAKE, dv=FAKE, cq=FAKE, ck=FAKE, ws=FAKE,
           wsb=1 << 30, B=2, Hq=8, Hkv=2, tq=100, tk=120, maxq=60, maxk=60, D=64, causal=0, scale=0.125, stream=None)


@pytest.mark.parametrize("change,expect", [
    ({"cq": None}, 1), ({"q": None}, 1), ({"dk": None}, 1), ({"tq": -1}, 1), ({"maxk": -1}, 1), ({"B": 0}, 1), ({"causal": -1}, 1),
    ({"D": 32}, 2), ({"tq": (1 << 31) - 1, "Hq": 512}, 2), ({"ck": FAKE + 2}, 3), ({"o": FAKE + 4}, 3), ({"wsb": 0}, 4)])
def test_attn_bwd_varlen_rejects(lib, change, expect):
    assert _caller(lib.loom_attn_bwd_varlen, VAR)(**change) == expect


def test_attn_bwd_varlen_without_tokens(lib):
    call = _caller(lib.loom_attn_bwd_varlen, VAR)
    none = dict(do=None, q=None, o=None, lse=None, dq=None)
    assert call(tq=0, tk=0, k=None, v=None, dk=None, dv=None, ws=None, **none) == 0


def test_bwd_workspace_sizes(lib):
    # the row statistics of every query, and nothing on invalid sizes
    need = lib.loom_attn_bwd_workspace_bytes
    assert need(2, 8, 2, 300, 300, 64) >= 2 * 8 * 300 * 8
    assert need(1, 8, 1, 4096, 4096, 128) > need(64, 8, 1, 64, 64, 128)  # few long items are split
    assert need(2, 8, 3, 300, 300, 64) == 0 and need(2, 8, 2, 300, 300, 80) == 0 and need(2, 8, 2, 0, 300, 64) == 0
    var = lib.loom_attn_bwd_varlen_workspace_bytes
    assert var(5, 8, 2, 300, 300, 64) >= 8 * 300 * 8 and var(5, 8, 2, 0, 0, 64) > 0 and var(0, 8, 2, 3, 3, 64) == 0


NORM = dict(qkv=FAKE, stride=12 * 64, qw=FAKE, kw=FAKE, wt=0, cos=FAKE, sin=FAKE, P=100, R=64, inter=0, pos=None)
FWD = dict(NORM, q=FAKE, k=FAKE, v=FAKE, T=6, S=3, Hq=8, Hkv=2, D=64, eps=1e-6, stream=None)
SHARED = [
    ({"qkv": None}, 1), ({"kw": None}, 1), ({"sin": None}, 1), ({"T": -1}, 1), ({"P": 0}, 1), ({"Hkv": 0}, 1), ({"wt": 2}, 1),
    ({"inter": 3}, 1), ({"eps": 0.0}, 1), ({"eps": float("nan")}, 1), ({"stride": 12 * 64 - 8}, 1), ({"D": 96}, 2), ({"R": 24}, 2),
    ({"R": 0}, 2), ({"R": 80}, 2), ({"stride": 12 * 64 + 4}, 3), ({"qkv": FAKE + 8}, 3), ({"cos": FAKE + 4}, 3),
    ({"pos": FAKE + 2}, 3)]


@pytest.mark.parametrize("change,expect", SHARED + [({"q": None}, 1), ({"S": 4}, 1), ({"S": -1}, 1), ({"v": FAKE + 8}, 3)])
def test_norm_rope_rejects(lib, change, expect):
    assert _caller(lib.loom_qkv_norm_rope, FWD)(**change) == expect


CACHE = dict(NORM, pos=FAKE, slots=FAKE, q=FAKE, kc=FAKE, vc=FAKE, pages=10, page=16, layout=0, T=6, Hq=8, Hkv=2, D=64, eps=1e-6,
             stream=None)


@pytest.mark.parametrize("change,expect", SHARED + [
    ({"pos": None}, 1), ({"slots": None}, 1), ({"kc": None}, 1), ({"pages": 0}, 1), ({"page": 0}, 1), ({"layout": 2}, 1),
    ({"pages": 1 << 20, "page": 1 << 12}, 2), ({"slots": FAKE + 1}, 3), ({"vc": FAKE + 8}, 3)])
def test_norm_rope_cache_rejects(lib, change, expect):
    assert _caller(lib.loom_qkv_norm_rope_cache, CACHE)(**change) == expect


NBWD = dict(dq=FAKE, dk=FAKE, dv=FAKE, **NORM, dqkv=FAKE, dstride=12 * 64, dqw=FAKE, dkw=FAKE, ws=FAKE, wsb=1 << 30, T=6, S=0, Hq=8,
            Hkv=2, D=64, eps=1e-6, stream=None)


@pytest.mark.parametrize("change,expect", SHARED + [
    ({"dq": None}, 1), ({"dqkv": None}, 1), ({"dkw": None}, 1), ({"S": 4}, 1), ({"dstride": 64}, 1), ({"dstride": 12 * 64 + 2}, 3),
    ({"dqw": FAKE + 2}, 3), ({"ws": None}, 4), ({"wsb": 64}, 4), ({"ws": FAKE + 8}, 3)])
def test_norm_rope_bwd_rejects(lib, change, expect):
    assert _caller(lib.loom_qkv_norm_rope_bwd, NBWD)(**change) == expect


def test_nothing_to_do(lib):
    assert _caller(lib.loom_qkv_norm_rope, FWD)(T=0, S=0) == 0
    assert _caller(lib.loom_qkv_norm_rope_cache, CACHE)(T=0) == 0
    assert lib.loom_qkv_norm_rope_bwd_workspace_bytes(96) == 0


def test_norm_backward_heads(lib):
    """More heads than the gradient's warps can be dealt to, by their rows' length."""
    assert _caller(lib.loom_qkv_norm_rope_bwd, NBWD)(Hq=16384, Hkv=1, stride=16386 * 64, dstride=16386 * 64) == 2
