"""Rotation tables with fewer rows than the implied positions need: refused, forward and backward."""
import pytest

from tests.test_abi_grad import FWD, NBWD, _caller, lib  # noqa: F401


@pytest.mark.parametrize("T,S,P", [(6, 0, 5), (6, 3, 2), (1 << 20, 1 << 20, 1 << 19), (4, 4, 3)])
def test_abi_refuses_short_tables(lib, T, S, P):  # noqa: F811
    assert _caller(lib.loom_qkv_norm_rope, FWD)(T=T, S=S, P=P) == 1
    assert _caller(lib.loom_qkv_norm_rope_bwd, NBWD)(T=T, S=S, P=P) == 1


def test_no_tokens_need_no_rows(lib):  # noqa: F811
    assert _caller(lib.loom_qkv_norm_rope, FWD)(T=0, S=500, P=1) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["compiled", "python"])
def test_the_binding_names_short_tables(monkeypatch, way):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    import paper_2609_29219_gb300 as loom
    loom._torch()
    if way == "python":
        monkeypatch.setattr(loom, "_fast", None)
    z = lambda *s: torch.zeros(s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    tables = torch.rand((2, 5, 32), device="cuda")
    args = (torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), tables[0], tables[1])
    for T, S, fits in ((6, 0, False), (12, 6, False), (5, 0, True), (10, 5, True)):
        shape = lambda h: (T // S, h, S, 64) if S else (T, h, 64)  # noqa: B023, E731
        calls = (lambda: loom.loom_qkv_norm_rope(z(T, 256), *args, 2, 1, seq_len=S),  # noqa: B023
                 lambda: loom.loom_qkv_norm_rope_bwd(z(*shape(2)), z(*shape(1)), z(*shape(1)), z(T, 256), *args))  # noqa: B023
        for f in calls:
            if fits:
                f()
            else:
                with pytest.raises(ValueError, match="cos and sin"):
                    f()
    # positions on the device are the caller's: clamped
    loom.loom_qkv_norm_rope(z(6, 256), *args, 2, 1, torch.arange(6, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
