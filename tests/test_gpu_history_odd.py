"""GPU: infinities and NaN in keys that rows do see: a NaN score makes the row NaN and no other, a
score of minus infinity is a weight of zero, whatever the kernel's width makes of it inside."""

import numpy as np
import pytest
import torch

from oracle import history as oracle
from paper_2607_27744_amd import ops
from test_gpu_history import BF, F32, _case, _np, _off, check

pytestmark = pytest.mark.gpu

WIDTHS = [(BF, 64), (BF, 128), (BF, 24), (BF, 100), (F32, 32), (F32, 40), (F32, 5), (F32, 256)]


@pytest.mark.parametrize("dtype, d", WIDTHS)
@pytest.mark.parametrize("cap", [0.0, 20.0, 1e4])
@pytest.mark.parametrize("new", [[200, 90, 400], [1, 40, 3], [1, 2, 1]])
def test_nan_scores(gpu_lib, dtype, d, cap, new):
    lens = [200, 90, 1300]
    q, k, v = _case(dtype, 4, 2, d, new, lens, seed=d)
    want = oracle.attention(_np(q), _np(k), _np(v), new, lens, cap=cap)
    at = 150                                     # a key of the first request
    k[at, 1] = float("nan")                      # of its second K/V head
    pos = 200 - new[0] + np.arange(new[0])
    hit = np.zeros((sum(new), 4), bool)
    hit[:new[0], 2:] = (pos >= at)[:, None]
    got = ops.history_attention(q, k, v, _off(new), _off(lens), cap=cap)
    assert bool(torch.isnan(got[torch.from_numpy(hit)]).all()) and hit.any()
    ok = ~hit
    check(got[torch.from_numpy(ok)], *(x[ok] for x in want), 1300, "bf16" if dtype == BF else "fp32")


@pytest.mark.parametrize("dtype, d", WIDTHS)
@pytest.mark.parametrize("most", [None, 64])
@pytest.mark.parametrize("new", [130, 2])
def test_scores_of_minus_infinity(gpu_lib, dtype, d, most, new):
    # One dim of a key at minus infinity, where every query is positive: the key has no weight.
    q, k, v = _case(dtype, 2, 1, d, [new], [700], seed=d)
    for dim in (0, d - 1):
        x, y = q.clone(), k.clone()
        x[:, :, dim] = x[:, :, dim].abs() + 0.1
        y[300, :, dim] = -float("inf")
        got = ops.history_attention(x, y, v, _off([new]), _off([700]), causal=False, max_kv_len=most)
        keep = np.arange(700) != 300
        want = oracle.attention(_np(x), _np(k)[keep], _np(v)[keep], [new], [699], causal=False)
        check(got, *want, 700, "bf16" if dtype == BF else "fp32")
