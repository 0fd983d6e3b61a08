"""GPU: rows that are asked for on top of what a slot holds, past 32 bits together: refused like any
other number that its table row has no room for, with nothing read by it or changed."""

import pytest
import torch

from gpu_util import dev_i32
from paper_2607_27744_amd import ops

pytestmark = pytest.mark.gpu

TOP = 2 ** 31 - 1


@pytest.mark.parametrize("page", [1, 2, 4, 1000])
@pytest.mark.parametrize("length, rows", [(TOP, TOP), (TOP, 1), (5, TOP), (0, TOP), (TOP, 0)])
def test_sums_past_32_bits(gpu_lib, page, length, rows):
    pool, table, lens, refs = ops.cache_pool(1, 6, page, 1, 4, slots=3, table_width=2)
    lens[1] = length
    kept = [t.clone() for t in (table, lens, refs)]
    for padded in (8, 5000):              # places found by the first launch, by the second
        got, status = ops.cache_reserve(dev_i32([1]), dev_i32([0, rows]), padded, table, lens, refs,
                                        page)
        assert status.tolist() == [2, 0] and bool((got == -1).all())
        assert all(torch.equal(a, b) for a, b in zip(kept, (table, lens, refs)))


def test_the_last_row_that_fits(gpu_lib):
    pool, table, lens, refs = ops.cache_pool(1, 6, 4, 1, 4, slots=3, table_width=2)
    for add, code in ((5, 0), (4, 2), (3, 0), (1, 2), (0, 0)):
        _, status = ops.cache_reserve(dev_i32([1]), dev_i32([0, add]), add, table, lens, refs, 4)
        assert status[0].item() == code
    assert lens.tolist() == [0, 8, 0]
