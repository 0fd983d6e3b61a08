"""One workspace for history attention calls of many sizes: the bound that include/rocs_history.h
states, against the sizes of single calls, which are not monotone."""

import numpy as np
import pytest
import torch

from gpu_util import dev_i32
from paper_2607_27744_amd import _lib, ops
from test_history_abi import P, _paged, lib, no_gpu   # noqa: F401 (lib: a fixture)


def bound(rows, heads, head_dim, most, bf16):
    c = 524288 if bf16 and head_dim % 8 == 0 and head_dim <= 128 else 8192
    return 4 * (head_dim + 2) * min(heads * rows * min(256, -(-most // 256)), c) + 512


def test_sizes_are_a_calls_own(lib):   # noqa: F811
    size = lib.rocs_history_workspace_size
    assert size(2048, 2048, 8, 8, 128, 4096, 1) < size(512, 512, 8, 8, 128, 4096, 1)
    assert size(1, 1, 8, 1, 128, 66000, 1) < size(1, 1, 8, 1, 128, 65536, 1)


def test_the_bound_covers_every_call(lib):   # noqa: F811
    rng = np.random.default_rng(0)
    size, tight = lib.rocs_history_workspace_size, 0.0

    def log(lo, hi):
        return int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
    for _ in range(40000):
        hk = int(rng.choice([1, 2, 3, 4, 8, 16]))
        h, d = hk * int(rng.choice([1, 2, 4, 8])), int(rng.choice([5, 8, 64, 100, 128, 129, 256]))
        r, n, most, bf16 = log(1, 5000), log(1, 100000), log(1, 300000), int(rng.integers(2))
        need = size(r, n, h, hk, d, most, bf16)
        # ... and so every call of at most n rows and `most` keys, as it grows with both.
        limit = bound(n, h, d, most, bf16)
        assert need <= limit
        assert limit <= bound(n + log(1, 5000), h, d, most + log(1, 5000), bf16)
        tight = max(tight, need / limit)
    assert tight > 0.5


@no_gpu
def test_paged_sizes_follow_the_table(lib):   # noqa: F811
    # 16 pages of 64 rows: a looser bound on the lengths than the table's plans no other parts.
    kw = dict(W=16, page=64, P=200, R=1, N=1, S=1, H=8, Hk=8, D=128, ws=P(0x90000000))
    need = lib.rocs_history_workspace_size(1, 1, 8, 8, 128, 16 * 64, 1)
    assert need > 0
    for most in (0, 1024, 100000):
        assert _paged(lib, most=most, ws_bytes=need - 1, **kw) == _lib.WORKSPACE_TOO_SMALL
        assert _paged(lib, most=most, ws_bytes=need, **kw) not in (_lib.OK, _lib.WORKSPACE_TOO_SMALL,
                                                                   _lib.INVALID_ARGUMENT)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d", [(torch.bfloat16, 128), (torch.bfloat16, 40), (torch.float32, 64)])
def test_one_workspace_for_all_batches(gpu_lib, dtype, d):
    h, hk, most, n_most = 8, 4, 5000, 300
    need = bound(n_most, h, d, most, dtype == torch.bfloat16)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    for rows, lens in (([1], [5000]), ([150, 150], [5000, 300]), ([1] * 30, [170] * 30), ([5], [700]),
                       ([1] * 300, [16] * 300), ([32, 33], [2500, 2400])):
        q = torch.randn((sum(rows), h, d), device="cuda", generator=g).to(dtype)
        k, v = (torch.randn((sum(lens), hk, d), device="cuda", generator=g).to(dtype) for _ in range(2))
        qo, ko = (dev_i32(np.concatenate([[0], np.cumsum(x)])) for x in (rows, lens))
        for bound_len in (max(lens), most):
            got = ops.history_attention(q, k, v, qo, ko, max_kv_len=bound_len, workspace=ws)
            assert torch.equal(got, ops.history_attention(q, k, v, qo, ko, max_kv_len=bound_len))
