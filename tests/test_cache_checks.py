"""What the cache's entry points in ops.py refuse, beside test_history_abi's (no GPU needed)."""

import pytest
import torch

from paper_2607_27744_amd import ops


def test_cache_copy_refuses_what_is_no_pool():
    pages = torch.zeros(1, dtype=torch.int32)
    pool = torch.zeros(2, 3, 4, 8)
    for bad in (torch.zeros(()), torch.zeros(8), pool[0], pool.transpose(0, 1), pool[:, :0]):
        for args in ((bad,), (pool, bad)):
            with pytest.raises(ValueError, match="pool must be"):
                ops.cache_copy(pages, pages, *args)
    with pytest.raises(ValueError, match="same layers"):
        ops.cache_copy(pages, pages, pool, torch.zeros(2, 3, 2, 8))
    with pytest.raises(ValueError, match="on the GPU"):
        ops.cache_copy(pages, pages, pool)
