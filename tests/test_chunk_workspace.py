"""The bound that the header gives for the chunk attention's workspace (no GPU needed)."""
import itertools

import pytest


@pytest.fixture(scope="module")
def loom():
    from paper_2609_29219_gb300 import build
    build.build()
    import paper_2609_29219_gb300 as m
    return m


def test_the_bound_is_reached_and_kept(loom):
    try:
        import torch
        sms = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 152
    except ImportError:
        sms = 152
    most = 0
    for (Hq, Hkv), T, D in itertools.product(((1, 1), (32, 8), (32, 32), (64, 1), (6, 3), (130, 1), (131, 1), (65536, 1)),
                                             (1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 5000, 32767), (64, 128)):
        most = max(most, loom.loom_attn_chunk_paged_workspace_bytes(1, Hq, Hkv, T, D))
    assert most == 16384 + 266240 * min(sms, 256)
