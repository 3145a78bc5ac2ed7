"""Counts of page moves that no array has (no GPU): twice such a count leaves 64 bits, and the moves went unchecked."""
import pytest
import torch

from paper_2511_10909_amd import binding as mm


@pytest.mark.parametrize("count", [2 ** 32 + 1, 2 ** 63, 2 ** 63 + 1, 2 ** 64 - 1])
@pytest.mark.parametrize("layers", [0, 1])
def test_a_count_beyond_any_array_is_refused(count, layers):
    moves = torch.tensor([[0, 1]], dtype=torch.int32)
    assert mm._lib.mmaemu_cache_copy_pages(1 << 20, moves.data_ptr(), count, 10, 160, layers, 0, None) == 3
    assert "count" in mm.last_error()
