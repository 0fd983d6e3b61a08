"""GPU: capped scores over the whole range of caps. A cap far above the scores changes nothing that
counts, so its own rounding must not either: the oracle's bound on a score's error follows the
score there, not the cap. Tolerances are those of test_gpu_history."""

import numpy as np
import pytest
import torch

from oracle import history as oracle
from paper_2607_27744_amd import ops
from test_gpu_history import BF, F32, _call_kw, _case, _np, _off, _paged, check

pytestmark = pytest.mark.gpu

CAPS = [64.0, 128.0, 129.0, 1e3, 1e4, 1e6, 1e8, 1e30, 3e38]
SHAPES = [  # dtype, H, H_kv, d, query rows, history rows: tiles of 128 rows, of 32, fp32
    (BF, 2, 2, 64, [300, 70], [300, 70]), (BF, 4, 2, 128, [200, 65], [400, 129]),
    (BF, 4, 1, 128, [1, 3], [700, 90]), (BF, 2, 2, 64, [1, 2], [3000, 300]),
    (BF, 2, 1, 40, [90, 1], [200, 1]), (F32, 2, 1, 64, [40, 3], [200, 3])]
RULES = {"causal": dict(), "full": dict(causal=False),
         "slope": dict(slopes=np.array([0.25, 0.5, 0.1, 0.01], np.float32))}


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("rule", list(RULES))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{str(s[0])[6:]}-{s[1]}.{s[2]}x{s[3]}-{s[4][0]}")
def test_any_cap(gpu_lib, shape, rule, cap):
    dtype, h, hk, d, q_len, kv_len = shape
    kw = dict(RULES[rule], cap=cap)
    if "slopes" in kw:
        kw["slopes"] = kw["slopes"][:h]
    what = "bf16" if dtype == BF else "fp32"
    for std in (1.0, 6.0):                # scores of units, and of hundreds (past a quarter of a cap)
        q, k, v = _case(dtype, h, hk, d, q_len, kv_len, seed=d, std=std)
        want = oracle.attention(_np(q), _np(k), _np(v), q_len, kv_len, **kw)
        got = ops.history_attention(q, k, v, _off(q_len), _off(kv_len), **_call_kw(kw))
        check(got, *want, max(kv_len), what)
        pool, table, lens, slots = _paged(k, v, kv_len, 16)
        got = ops.paged_attention(q, pool[:, :, 0], pool[:, :, 1], table, lens, _off(q_len), slots=slots,
                                  **_call_kw(kw))
        check(got, *want, max(kv_len), what)


@pytest.mark.parametrize("cap", [129.0, 1e6, 1e30])
@pytest.mark.parametrize("d", [64, 128])
def test_any_cap_with_documents(gpu_lib, d, cap):
    lens = [700, 130]
    q, k, v = _case(BF, 2, 2, d, lens, lens, seed=d)
    docs = np.concatenate([np.arange(n) // 150 for n in lens])
    for extra in (dict(), dict(slopes=np.array([0.1, 0.02], np.float32)), dict(prefix=np.array([90, 200]))):
        kw = dict(extra, cap=cap, q_docs=docs, kv_docs=docs)
        got = ops.history_attention(q, k, v, _off(lens), _off(lens), **_call_kw(kw))
        check(got, *oracle.attention(_np(q), _np(k), _np(v), lens, lens, **kw), max(lens), "bf16")


@pytest.mark.parametrize("cap", [1e6, 1e30])
def test_a_far_cap_is_no_cap(gpu_lib, cap):
    # The two results differ by no more than each may from the definition.
    lens = [512]
    for new in ([512], [1]):
        q, k, v = _case(BF, 2, 2, 128, new, lens, seed=1)
        call = lambda c: ops.history_attention(q, k, v, _off(new), _off(lens), cap=c)  # noqa: E731
        want, mean, err = oracle.attention(_np(q), _np(k), _np(v), new, lens, cap=cap)
        check(call(cap), _np(call(0.0)), 2 * mean, 2 * err, 512, "bf16")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_small_caps_and_large_scales(gpu_lib, dtype):
    # Scores of nothing, or past the type's range, meet a factor that is finite: the weights are equal.
    lens = [200]
    for new in ([200], [2]):
        q, k, v = _case(dtype, 2, 2, 64, new, lens, seed=2)
        k[::3] = 0
        got = ops.history_attention(q, k, v, _off(new), _off(lens), cap=1e-30, scale=1e12)
        n = 200 - new[0] + np.arange(new[0]) + 1
        sums = np.cumsum(_np(v), 0)[n - 1] / n[:, None, None]
        mean = np.cumsum(np.abs(_np(v)), 0)[n - 1] / n[:, None, None]
        check(got, sums, mean, np.zeros(mean.shape[:2]), 200, "bf16" if dtype == BF else "fp32")
