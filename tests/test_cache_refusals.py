"""What the key/value cache's binding and library refuse beyond the common mistakes (no GPU needed)."""
import pytest
import torch

from paper_2202_07471_b200 import cache

I32 = torch.int32


def parts(batch=3, width=2):
    return torch.zeros(batch, dtype=I32), torch.zeros((batch, width), dtype=I32), torch.zeros(batch + 1, dtype=I32)


@pytest.mark.parametrize("shape", [(4, 0, 4, 1152), (4, 2, 0, 1152), (0, 0, 0, 1152)])
def test_a_cache_without_heads_or_positions_is_refused(shape):
    with pytest.raises(ValueError, match="cache"):
        cache._cache_rows(torch.zeros(shape, dtype=torch.uint8), *parts(), 5)
    assert cache._cache_rows(torch.zeros((0, 2, 4, 1152), dtype=torch.uint8), *parts(), 5).page_count == 0   # no pages: everything counts as not there
