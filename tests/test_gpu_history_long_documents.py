"""GPU: documents in histories of more 64-key stages than a tile lists (2,048): it walks them whole."""

import numpy as np
import pytest

from oracle import history as oracle
from paper_2607_27744_amd import ops
from test_gpu_history import BF, _call_kw, _case, _np, _off, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d, rule", [(64, dict()), (128, dict(slopes=np.array([0.001], np.float32))),
                                     (64, dict(causal=False, cap=30.0))])
@pytest.mark.parametrize("most", [64, None])
def test_more_stages_than_the_list(gpu_lib, d, rule, most):
    # 2,065 stages; a bound below them makes them one part, without one they are cut and listed.
    new, lens = [150, 3], [2065 * 64 - 17, 90]
    q, k, v = _case(BF, 1, 1, d, new, lens, seed=d)
    docs = np.concatenate([np.arange(lens[0]) // 9000, np.zeros(lens[1], int)])
    tail = np.concatenate([docs[lens[0] - new[0]:lens[0]], docs[-new[1]:]])
    tail[:40] = 3                                            # rows of an early document
    tail[40:50] = 99                                         # rows of none
    kw = dict(rule, q_docs=tail, kv_docs=docs)
    got = ops.history_attention(q, k, v, _off(new), _off(lens), max_kv_len=most, **_call_kw(kw))
    want = oracle.attention(_np(q), _np(k), _np(v), new, lens, **kw)
    check(got, *want, max(lens), "bf16")
    assert bool((got[40:50] == 0).all())
