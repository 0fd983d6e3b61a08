"""GPU: attention over packed and paged histories against the float64 oracle.

Tolerance per element, from the roundings that the kernels make: a score is off by at most e (the
oracle's bound), a softmax weight so by 2 e relative, by half a bf16 step (2^-8) where weights
are rounded for the matrix cores (numerator and row sum: twice), and the fp32 sums of L terms by
L 2^-24 each; all times the mean weight of |v|. The result is rounded once more."""

import numpy as np
import pytest
import torch

from gpu_util import dev_i32
from oracle import history as oracle
from paper_2607_27744_amd import ops

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _off(lens):
    return dev_i32(np.concatenate([[0], np.cumsum(lens)]))


def check(got, want, mean, err, longest, what=""):
    got = _np(got)
    bf = 2.0 ** -8 if what.startswith("bf16") else 0.0
    tol = mean * (2 * err[..., None] + 2 * bf + (2 * longest + 64) * oracle.U32)
    tol = tol + (bf if bf else oracle.U32) * (np.abs(want) + tol) + 1e-30
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off / tol), off.shape)
    assert np.all(off <= tol), f"{what}: {off[worst]:.3g} off at {worst}, {tol[worst]:.3g} allowed"


def _case(dtype, h, hk, d, q_len, kv_len, seed=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    n, m = int(np.sum(q_len)), int(np.sum(kv_len))
    mk = lambda rows, heads: (torch.randn(rows, heads, d, generator=g) * std).to(dtype).cuda()  # noqa: E731
    return mk(n, h), mk(m, hk), mk(m, hk)


def _rules(name, h, q_len, kv_len, seed=0):
    rng = np.random.default_rng(seed)
    kw = {"causal": dict(), "full": dict(causal=False), "cap": dict(cap=5.0),
          "slope": dict(slopes=np.float32(2.0) ** -np.arange(1, h + 1, dtype=np.float32)),
          "prefix": dict(prefix=np.array([n // 3 if i % 3 else n + 5 for i, n in enumerate(kv_len)])),
          "all": dict(cap=3.0, slopes=np.full(h, 0.01, np.float32),
                      prefix=np.array([n // 2 - 1 for n in kv_len]))}.get(name.split("-")[0], {})
    if "docs" in name:
        n, m = int(np.sum(q_len)), int(np.sum(kv_len))
        if "random" in name:          # any order; some query documents have no key at all
            kw = dict(kw, q_docs=rng.integers(0, 9, n), kv_docs=rng.integers(0, 7, m))
        else:
            docs = np.concatenate([np.sort(rng.integers(0, 1 + x // 60, x)) for x in kv_len])
            own = np.split(docs, np.cumsum(kv_len)[:-1])
            tail = np.concatenate([np.concatenate([np.full(max(a - x.size, 0), -7), x[x.size - min(a, x.size):]])
                                   for a, x in zip(q_len, own)])       # -7: a row before the history
            kw = dict(kw, q_docs=tail, kv_docs=docs)
    return kw


def _call_kw(kw):
    out = {k: v for k, v in kw.items() if k in ("causal", "cap")}
    if "prefix" in kw:
        out["prefix_lens"] = dev_i32(kw["prefix"])
    if "slopes" in kw:
        out["slopes"] = torch.from_numpy(kw["slopes"]).cuda()
    for k in ("q_docs", "kv_docs"):
        if k in kw:
            out[k] = dev_i32(kw[k])
    return out


SHAPES = [  # dtype, H, H_kv, d, query rows, history rows
    (BF, 4, 4, 64, [1, 63, 200, 0, 129], [1, 63, 200, 0, 129]),
    (BF, 4, 2, 128, [1, 7, 130, 1], [300, 64, 130, 65]),
    (BF, 8, 1, 64, [1, 1, 1, 1], [700, 1, 33, 512]),
    (BF, 2, 2, 128, [5, 40, 3], [3, 40, 0]),                 # more rows than history
    (F32, 2, 2, 32, [20, 31, 1, 0, 47], [20, 31, 1, 0, 47]),
    (F32, 6, 3, 80, [1, 17, 3], [90, 17, 200]),
    (BF, 3, 1, 40, [33, 2], [33, 150]),
    (F32, 1, 1, 5, [9, 1], [9, 4]), (F32, 2, 1, 256, [4], [70]), (BF, 1, 1, 129, [4], [70]),
]
RULES = ["causal", "full", "cap", "slope", "prefix", "all", "causal-docs", "full-docs-random",
         "all-docs"]


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{str(s[0])[6:]}-{s[1]}.{s[2]}x{s[3]}")
def test_packed_against_oracle(gpu_lib, shape, rule):
    dtype, h, hk, d, q_len, kv_len = shape
    q, k, v = _case(dtype, h, hk, d, q_len, kv_len, seed=d + len(rule))
    kw = _rules(rule, h, q_len, kv_len)
    got = ops.history_attention(q, k, v, _off(q_len), _off(kv_len), **_call_kw(kw))
    want = oracle.attention(_np(q), _np(k), _np(v), q_len, kv_len, **kw)
    check(got, *want, max(kv_len), "bf16" if dtype == BF else "fp32")


@pytest.mark.parametrize("requests, hk", [(1, 1), (3, 1), (16, 1), (17, 1), (1, 2), (4, 2), (5, 2),
                                          (1, 4), (3, 4), (6, 4), (9, 4), (1, 3), (5, 8)])
def test_tiles_over_the_dies(gpu_lib, requests, hk):
    # Few requests and K/V heads, where a head's tiles are dealt out in more than one way.
    lens = [40 + (37 * r) % 230 for r in range(requests)]
    q, k, v = _case(BF, 2 * hk, hk, 64, lens, lens, seed=requests)
    got = ops.history_attention(q, k, v, _off(lens), _off(lens))
    check(got, *oracle.attention(_np(q), _np(k), _np(v), lens, lens), max(lens), "bf16")


def _paged(k, v, kv_len, page, seed=0, spare=5, slots=None, fill=0.0):
    """The packed K/V of each request in shuffled pages: (pool, table, lens, slots)."""
    rng = np.random.default_rng(seed)
    hk, d = k.shape[1:]
    used = [-(-n // page) for n in kv_len]
    pages, width = sum(used) + spare, max(max(used), 1) + 2
    slots = rng.permutation(len(kv_len)) if slots is None else slots
    pool = torch.full((pages, page, 2, hk, d), fill, dtype=k.dtype, device="cuda")
    table = np.full((len(kv_len), width), -1, np.int64)
    lens = np.zeros(len(kv_len), np.int64)
    order, at, row = rng.permutation(pages), 0, 0
    for r, n in enumerate(kv_len):
        s = slots[r]
        lens[s] = n
        table[s, :used[r]] = order[at:at + used[r]]
        for i in range(0, n, page):
            p, m = int(order[at + i // page]), min(page, n - i)
            pool[p, :m, 0] = k[row + i:row + i + m]
            pool[p, :m, 1] = v[row + i:row + i + m]
        at += used[r]
        row += n
    return pool, dev_i32(table), dev_i32(lens), dev_i32(slots)


@pytest.mark.parametrize("page", [16, 48, 64, 7, 1, 256])
@pytest.mark.parametrize("rule", ["causal", "full", "cap", "slope", "prefix", "all"])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[2], SHAPES[3], SHAPES[5]],
                         ids=lambda s: f"{str(s[0])[6:]}-{s[1]}.{s[2]}x{s[3]}")
def test_paged_against_oracle(gpu_lib, shape, rule, page):
    dtype, h, hk, d, q_len, kv_len = shape
    q, k, v = _case(dtype, h, hk, d, q_len, kv_len, seed=page)
    kw = _rules(rule, h, q_len, kv_len)
    # What a page holds past its history's end is not read.
    pool, table, lens, slots = _paged(k, v, kv_len, page, fill=float("nan"))
    got = ops.paged_attention(q, pool[:, :, 0], pool[:, :, 1], table, lens, _off(q_len), slots=slots,
                              **_call_kw(kw))
    want = oracle.attention(_np(q), _np(k), _np(v), q_len, kv_len, **kw)
    check(got, *want, max(kv_len), "bf16" if dtype == BF else "fp32")


LONG = [  # split histories: few rows, long keys
    (BF, 8, 2, 128, [1], [9000], 16), (BF, 4, 4, 64, [1, 1, 1], [5000, 1, 20000], 64),
    (BF, 8, 8, 128, [150, 33], [7000, 2100], 32), (F32, 4, 2, 64, [1, 2], [3000, 6001], 10),
    (BF, 16, 1, 64, [40], [12001], 128), (BF, 2, 2, 72, [3], [5000], 16)]


@pytest.mark.parametrize("most", ["bound", "none", "too small"])
@pytest.mark.parametrize("rule", ["causal", "all"])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: f"{str(s[0])[6:]}-{s[1]}.{s[2]}x{s[3]}")
def test_long_histories(gpu_lib, shape, rule, most):
    dtype, h, hk, d, q_len, kv_len, page = shape
    q, k, v = _case(dtype, h, hk, d, q_len, kv_len, seed=page)
    kw = _rules(rule, h, q_len, kv_len)
    want = oracle.attention(_np(q), _np(k), _np(v), q_len, kv_len, **kw)
    what = "bf16" if dtype == BF else "fp32"
    # A bound below the longest history costs speed, not keys.
    n = {"bound": max(kv_len), "none": None, "too small": 700}[most]
    pool, table, lens, slots = _paged(k, v, kv_len, page)
    got = ops.paged_attention(q, pool[:, :, 0], pool[:, :, 1], table, lens, _off(q_len), slots=slots,
                              max_kv_len=n, **_call_kw(kw))
    check(got, *want, max(kv_len), what)
    got = ops.history_attention(q, k, v, _off(q_len), _off(kv_len), max_kv_len=n, **_call_kw(kw))
    check(got, *want, max(kv_len), what)


def test_long_documents(gpu_lib):
    # Packed sessions in a long row: whole stretches of keys are passed over.
    lens = [5000, 3001]
    q, k, v = _case(BF, 2, 2, 64, lens, lens, seed=3)
    for rule in ("causal-docs", "full-docs", "all-docs", "causal-docs-random"):
        kw = _rules(rule, 2, lens, lens, seed=4)
        got = ops.history_attention(q, k, v, _off(lens), _off(lens), **_call_kw(kw))
        want = oracle.attention(_np(q), _np(k), _np(v), lens, lens, **kw)
        check(got, *want, max(lens), "bf16")


@pytest.mark.parametrize("dtype, d", [(BF, 64), (BF, 128), (BF, 24), (F32, 64)])
@pytest.mark.parametrize("std", [0.0, 30.0, 1e4])
def test_extreme_scores(gpu_lib, dtype, d, std):
    # Equal scores; scores far apart (one key has all the weight), either sign, rising along
    # the history so that the running maximum moves often.
    lens = [300, 70]
    q, k, v = _case(dtype, 2, 1, d, lens, lens, seed=9, std=1.0)
    k = (k.float() * std * torch.linspace(0.01, 1, k.shape[0], device="cuda")[:, None, None]).to(dtype)
    off = _off(lens)
    for kw in (dict(), dict(cap=50.0)):
        want = oracle.attention(_np(q), _np(k), _np(v), lens, lens, **kw)
        got = ops.history_attention(q, k, v, off, off, **kw)
        check(got, *want, 300, "bf16" if dtype == BF else "fp32")


@pytest.mark.parametrize("dtype, d", [(BF, 64), (BF, 128), (BF, 24), (F32, 32)])
@pytest.mark.parametrize("rows", ["all", "last"])
def test_unseen_keys_may_hold_anything(gpu_lib, dtype, d, rows):
    lens = [200, 90, 1300]
    new = lens if rows == "all" else [1, 40, 3]
    q, k, v = _case(dtype, 4, 2, d, new, lens, seed=5)
    rng = np.random.default_rng(5)
    docs = np.concatenate([np.sort(rng.integers(0, 5, n)) for n in lens])
    tail = np.concatenate([docs[sum(lens[:i + 1]) - a:sum(lens[:i + 1])] for i, a in enumerate(new)])
    bad = torch.from_numpy(np.flatnonzero(docs == 2)).cuda()
    kw = dict(q_docs=tail, kv_docs=docs)
    want = oracle.attention(_np(q), _np(k), _np(v), new, lens, **kw)
    mine = torch.from_numpy(tail == 2)
    for value in (float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).min):
        kb, vb = k.clone(), v.clone()
        kb[bad], vb[bad] = value, value
        got = ops.history_attention(q, kb, vb, _off(new), _off(lens), **_call_kw(kw))
        check(got[~mine], want[0][~mine], want[1][~mine], want[2][~mine], 1300,
              "bf16" if dtype == BF else "fp32")
        if not np.isfinite(value) and mine.any():
            assert not torch.isfinite(got[mine]).all()
    # After the row itself, under the causal mask.
    kb, vb = k.clone(), v.clone()
    kb[199], vb[199] = float("nan"), float("inf")
    got = ops.history_attention(q, kb, vb, _off(new), _off(lens))
    want = oracle.attention(_np(q), _np(k), _np(v), new, lens)
    keep = torch.ones(sum(new), dtype=torch.bool)
    keep[new[0] - 1] = False
    check(got[keep], want[0][keep], want[1][keep], want[2][keep], 1300,
          "bf16" if dtype == BF else "fp32")


def test_strides_and_given_outputs(gpu_lib):
    lens = [70, 200, 1]
    n, h, hk, d = sum(lens), 4, 2, 64
    for dtype, at in ((BF, 0), (BF, 8), (BF, 3), (F32, 1)):
        wide = torch.randn(n + 2, (h + 2 * hk) * d + 16, device="cuda").to(dtype)
        x = wide[1:-1, at:at + (h + 2 * hk) * d]
        q = x[:, :h * d].unflatten(1, (h, d))
        k = x[:, h * d:(h + hk) * d].unflatten(1, (hk, d))
        v = x[:, (h + hk) * d:].unflatten(1, (hk, d))
        off = _off(lens)
        out = torch.full((n + 2, h, d), 7.0, dtype=dtype, device="cuda")
        got = ops.history_attention(q, k, v, off, off, out=out[1:-1])
        assert got.data_ptr() == out[1:-1].data_ptr()
        assert bool((out[0] == 7).all()) and bool((out[-1] == 7).all())
        want = ops.history_attention(q.contiguous(), k.contiguous(), v.contiguous(), off, off)
        ref = oracle.attention(_np(q), _np(k), _np(v), lens, lens)
        check(got, *ref, 200, "bf16" if dtype == BF else "fp32")
        check(want, *ref, 200, "bf16" if dtype == BF else "fp32")


def test_rows_past_the_last_request_stay(gpu_lib):
    # A padded batch: rows behind the last request belong to nobody.
    lens = [30, 50]
    for dtype, d in ((BF, 64), (F32, 16)):
        q, k, v = _case(dtype, 2, 2, d, [100], [100])
        out = torch.full_like(q, 5.0)
        off = _off(lens)
        ops.history_attention(q, k, v, off, off, out=out)
        assert bool((out[80:] == 5).all())
        ref = oracle.attention(_np(q[:80]), _np(k[:80]), _np(v[:80]), lens, lens)
        check(out[:80], *ref, 50, "bf16" if dtype == BF else "fp32")


@pytest.mark.parametrize("dtype, d, rows", [(BF, 64, 1), (BF, 128, 90), (F32, 16, 3)])
def test_rows_past_the_last_request_of_a_split_history(gpu_lib, dtype, d, rows):
    # Long and short histories in one split call: partial results for some rows, the result at
    # once for others, nothing for the rows of no request.
    lens, new = [6000, 200, 9000], [rows, 1, rows]
    q, k, v = _case(dtype, 4, 2, d, [sum(new) + 5], [sum(lens)], seed=6)
    assert ops.history_workspace_size(3, sum(new) + 5, 4, 2, d, 9000, dtype) > 0
    out = torch.full_like(q, 5.0)
    ops.history_attention(q, k, v, _off(new), _off(lens), max_kv_len=9000, out=out)
    n = sum(new)
    assert bool((out[n:] == 5).all())
    ref = oracle.attention(_np(q[:n]), _np(k), _np(v), new, lens)
    check(out[:n], *ref, 9000, "bf16" if dtype == BF else "fp32")


def test_bad_pages_and_slots_stay_inside(gpu_lib):
    # Ids out of range act as the last page or slot, lengths as the nearest possible one.
    q, k, v = _case(BF, 2, 2, 64, [1, 1], [40, 33])
    pool, table, lens, slots = _paged(k, v, [40, 33], 16, slots=np.array([0, 1]))
    last = pool.shape[0] - 1
    pool[last] = 0.5
    for bad in (-1, 1 << 30, pool.shape[0]):
        t2, t3 = table.clone(), table.clone()
        t2[1, 1], t3[1, 1] = bad, last
        args = (q, pool[:, :, 0], pool[:, :, 1])
        off = _off([1, 1])
        assert torch.equal(ops.paged_attention(*args, t2, lens, off, slots=slots),
                           ops.paged_attention(*args, t3, lens, off, slots=slots))
    got = ops.paged_attention(*args, table, lens, off, slots=dev_i32([0, 99]))
    assert torch.equal(got, ops.paged_attention(*args, table, lens, off))
    long = torch.where(table < 0, torch.zeros_like(table), table)
    a = ops.paged_attention(*args, long, dev_i32([1 << 30, -5]), off)
    b = ops.paged_attention(*args, long, dev_i32([long.shape[1] * 16, 0]), off)
    assert torch.equal(a, b) and bool((a[1] == 0).all())


def test_large_offsets(gpu_lib):
    # A cache whose pages lie past 2^31 elements and 2^32 bytes.
    pages, page, hk, d = 140000, 64, 2, 64
    pool = torch.zeros((pages, page, 2, hk, d), dtype=BF, device="cuda")
    q, k, v = _case(BF, 4, hk, d, [1, 70], [130, 190], seed=2)
    table = dev_i32([[pages - 1, 3, pages - 2], [pages - 3, pages // 2, pages - 4]])
    for r, (a, n) in enumerate(((0, 130), (130, 190))):
        for c in range(-(-n // page)):
            m = min(page, n - c * page)
            p = int(table[r, c])
            pool[p, :m, 0] = k[a + c * page:a + c * page + m]
            pool[p, :m, 1] = v[a + c * page:a + c * page + m]
    got = ops.paged_attention(q, pool[:, :, 0], pool[:, :, 1], table, dev_i32([130, 190]),
                              _off([1, 70]))
    want = oracle.attention(_np(q), _np(k), _np(v), [1, 70], [130, 190])
    check(got, *want, 190, "bf16")


def test_capture_streams_and_shared_workspace(gpu_lib):
    q, k, v = _case(BF, 8, 2, 128, [1, 3], [3000, 5000], seed=1)
    qo, ko = _off([1, 3]), _off([3000, 5000])
    need = ops.history_workspace_size(2, 4, 8, 2, 128, 8000, BF)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = [ops.history_attention(q * s, k, v, qo, ko, workspace=ws) for s in (1, 2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ops.history_attention(q, k, v, qo, ko, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want[0])
    ins, outs, graphs = [q.clone(), q.clone() * 2], [torch.empty_like(q) for _ in range(2)], []
    torch.cuda.synchronize()
    for x, y in zip(ins, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.history_attention(x, k, v, qo, ko, workspace=ws, out=y)
        graphs.append(g)
    for _ in range(3):
        for g, y, w in zip(graphs, outs, want):
            y.zero_()
            g.replay()
            assert torch.equal(ops.history_attention(q, k, v, qo, ko), want[0])
            torch.cuda.synchronize()
            assert torch.equal(y, w)


def test_no_rows_and_no_keys(gpu_lib):
    q, k, v = _case(BF, 2, 2, 64, [3], [0])
    assert bool((ops.history_attention(q, k, v, _off([3]), _off([0])) == 0).all())
    e = ops.history_attention(q[:0], k, v, _off([0, 0]), _off([0, 0]))
    assert e.shape == (0, 2, 64)
    pool, table, lens, refs = ops.cache_pool(1, 4, 16, 2, 64, slots=2, table_width=2)
    out = ops.paged_attention(q, pool[0, :, :, 0], pool[0, :, :, 1], table, lens, _off([2, 1]))
    assert bool((out == 0).all())


def test_python_path_gives_the_same(gpu_lib, monkeypatch):
    q, k, v = _case(BF, 4, 2, 64, [5, 1], [90, 200])
    pool, table, lens, slots = _paged(k, v, [90, 200], 16)
    calls = [lambda: ops.history_attention(q, k, v, _off([5, 1]), _off([90, 200]), cap=20.0),
             lambda: ops.paged_attention(q, pool[:, :, 0], pool[:, :, 1], table, lens, _off([5, 1]),
                                         slots=slots, scale=0.1)]
    taken = [ops._native().history(q, k, v, _off([5, 1]), _off([90, 200]), True, None, None, None,
                                   None, 20.0, None, None, None, None, None),
             ops._native().paged(q, pool[:, :, 0], pool[:, :, 1], table, lens, _off([5, 1]), slots,
                                 True, None, None, 0.0, None, 0.1, None, None, None)]
    assert all(t is not None for t in taken)
    want = [c() for c in calls]
    monkeypatch.setattr(ops, "_binding", ops._PythonPath())
    for c, w, t in zip(calls, want, taken):
        assert torch.equal(c(), w) and torch.equal(t, w)
