"""The numbers of a step's bookkeeping: whole ones that fit, looked at before the tensors (no GPU needed)."""
import numpy as np
import pytest
import torch

import paper_2609_29219_gb300 as loom


def _plan(num_tokens, page_size):
    ints = torch.zeros(2, dtype=torch.int32)
    return loom.loom_paged_plan(ints, ints, ints.view(2, 1), ints, ints[:1], num_tokens, page_size)


@pytest.mark.parametrize("bad", [2.5, 16.0, np.float64(16), "16", None, torch.tensor(16.0), torch.tensor([16, 16])])
def test_what_is_no_whole_number_is_refused(bad):
    for args in ((bad, 16), (16, bad)):
        with pytest.raises(TypeError):
            _plan(*args)


def test_numbers_past_32_bits_are_refused():
    """Cut to 32 bits they would be others: 2^32 + 16 rows a page 16."""
    for args in ((1 << 31, 16), ((1 << 32) + 5, 16), (5, 1 << 31), (5, (1 << 32) + 16), (5, 16 - (1 << 32))):
        with pytest.raises(ValueError, match="2.31"):
            _plan(*args)
    with pytest.raises(ValueError, match="negative"):
        _plan(-1, 16)


@pytest.mark.parametrize("good", [16, np.int64(16), np.int32(16), torch.tensor(16)])
def test_whole_numbers_of_any_kind(good):
    with pytest.raises(ValueError, match="new_lens must be a CUDA tensor"):  # the next thing that is wrong
        _plan(good, good)
