"""GPU: attention over a cache held in 4 bits against the float64 oracle of the values that it holds.

Tolerance per element as for the other pools: a score is off by at most e (the oracle's bound), a
softmax weight so by 2 e relative, by half a bf16 step (2^-8) where weights are rounded for the matrix
cores (numerator and row sum: twice), and the fp32 sums of L terms by L 2^-24 each; all times the mean
weight of |v|. The result is rounded once more. (K and V themselves are exact in bf16.)"""

import numpy as np
import pytest
import torch

from gpu_util import dev_i32
from oracle import history as oracle
from oracle import layer
from paper_2607_27744_amd import ops

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def check(got, want, mean, err, longest, bf):
    got = _np(got)
    step = 2.0 ** -8 if bf else 0.0
    tol = mean * (2 * err[..., None] + 2 * step + (2 * longest + 64) * oracle.U32)
    tol = tol + (step if bf else oracle.U32) * (np.abs(want) + tol) + 1e-30
    assert np.all(np.isfinite(got)), "not finite"
    off = np.abs(got - want)
    worst = np.unravel_index(np.argmax(off / tol), off.shape)
    assert np.all(off <= tol), f"{off[worst]:.3g} off at {worst}, {tol[worst]:.3g} allowed"


def make(dtype, h, hk, d, q_len, kv_len, page, seed=0, spare=3):
    """(call arguments, K, V of the packed histories as the cache holds them). Pages and slots in any
    order; what no history holds is filled with scales of 255 (NaN)."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    m = int(np.sum(kv_len))
    codes = rng.integers(0, 16, (m, 2, hk, d)).astype(np.uint8)
    scale = rng.integers(124, 128, (m, 2, hk, d // 32)).astype(np.uint8)
    rows = np.zeros((m, layer.row_bytes(hk, d)), np.uint8)
    flat = codes.reshape(m, -1)
    rows[:, :hk * d] = flat[:, 0::2] | flat[:, 1::2] << 4
    rows[:, hk * d:hk * d + hk * d // 16] = scale.reshape(m, -1)
    kv = layer.unpack(rows, hk, d)
    used = [-(-n // page) for n in kv_len]
    pages = sum(used) + spare
    ids = rng.permutation(pages)
    slots = rng.permutation(len(kv_len) + 2)[:len(kv_len)]
    table = np.full((len(kv_len) + 2, max(max(used), 1) + 1), -1)
    lens = np.zeros(len(kv_len) + 2, int)
    pool = np.full((pages, page, rows.shape[1]), 0xff, np.uint8)
    at = row = 0
    for s, n, u in zip(slots, kv_len, used):
        table[s, :u], lens[s] = ids[at:at + u], n
        for j in range(u):
            part = rows[row + j * page:row + min((j + 1) * page, n)]
            pool[ids[at + j], :part.shape[0]] = part
        at += u
        row += n
    q = torch.randn(int(np.sum(q_len)), h, d, generator=g).to(dtype).cuda()
    call = dict(q=q, pages=torch.from_numpy(pool).cuda(), page_table=dev_i32(table), kv_lens=dev_i32(lens),
                q_offsets=dev_i32(np.concatenate([[0], np.cumsum(q_len)])), kv_heads=hk, slots=dev_i32(slots))
    return call, kv[:, 0], kv[:, 1]


def rules(name, h, kv_len):
    return {"causal": dict(), "full": dict(causal=False), "cap": dict(cap=5.0), "wide": dict(cap=300.0),
            "slope": dict(slopes=np.float32(2.0) ** -np.arange(1, h + 1, dtype=np.float32)),
            "prefix": dict(prefix=np.array([n // 3 if i % 3 else n + 5 for i, n in enumerate(kv_len)])),
            "all": dict(cap=3.0, slopes=np.full(h, 0.01, np.float32),
                        prefix=np.array([n // 2 - 1 for n in kv_len])),
            "all-wide": dict(cap=500.0, slopes=np.full(h, 0.02, np.float32))}[name]


def call_kw(kw):
    out = {k: v for k, v in kw.items() if k in ("causal", "cap")}
    if "prefix" in kw:
        out["prefix_lens"] = dev_i32(kw["prefix"])
    if "slopes" in kw:
        out["slopes"] = torch.from_numpy(kw["slopes"]).cuda()
    return out


SHAPES = [  # dtype, H, H_kv, d, page, query rows, history rows
    (BF, 8, 2, 128, 16, [1], [300]), (BF, 4, 4, 64, 64, [1, 1, 1, 1], [700, 1, 33, 512]),
    (BF, 8, 8, 128, 32, [1, 1, 1], [257, 64, 1025]), (BF, 3, 1, 128, 7, [1, 1], [90, 8]),
    (BF, 16, 1, 64, 24, [1, 2, 1], [129, 400, 3]),                        # up to 32 rows a head
    (BF, 4, 2, 128, 16, [1, 7, 130, 0, 1], [300, 64, 130, 20, 65]),
    (BF, 4, 4, 64, 48, [63, 200, 129], [63, 500, 129]),                   # chunks
    (BF, 2, 1, 128, 11, [90, 40], [700, 41]), (BF, 8, 2, 32, 16, [1, 40], [200, 90]),
    (BF, 6, 3, 96, 16, [1, 1, 50], [70, 200, 333]), (BF, 2, 2, 96, 5, [1, 9], [99, 40]),
    (BF, 2, 2, 128, 16, [5, 40, 3], [3, 40, 0]),                          # more rows than history
    (BF, 2, 1, 160, 16, [4], [70]), (BF, 2, 1, 256, 16, [1, 3], [70, 200]),
    (F32, 2, 2, 32, 16, [20, 31, 1, 0, 47], [20, 31, 1, 0, 47]), (F32, 6, 3, 96, 9, [1, 17, 3], [90, 17, 200]),
    (F32, 8, 1, 64, 16, [1, 1], [400, 31]), (F32, 4, 2, 128, 64, [1, 30], [600, 90]),
    (F32, 1, 1, 224, 16, [4], [70]),
]
RULES = ["causal", "full", "cap", "wide", "slope", "prefix", "all", "all-wide"]


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("shape", SHAPES,
                         ids=lambda s: f"{str(s[0])[6:]}-{s[1]}.{s[2]}x{s[3]}p{s[4]}n{sum(s[5])}")
def test_against_oracle(gpu_lib, shape, rule):
    dtype, h, hk, d, page, q_len, kv_len = shape
    call, k, v = make(dtype, h, hk, d, q_len, kv_len, page, seed=d + len(rule))
    kw = rules(rule, h, kv_len)
    got = ops.paged_attention_fp4(**call, **call_kw(kw))
    check(got, *oracle.attention(_np(call["q"]), k, v, q_len, kv_len, **kw), max(kv_len), dtype == BF)


@pytest.mark.parametrize("length", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257,
                                    511, 513, 1023, 1025, 2049])
@pytest.mark.parametrize("h, hk, d", [(8, 8, 128), (8, 1, 64), (4, 2, 128)])
def test_lengths(gpu_lib, h, hk, d, length):
    kv_len = [length, 40]
    call, k, v = make(BF, h, hk, d, [1, 1], kv_len, 16, seed=length)
    want = oracle.attention(_np(call["q"]), k, v, [1, 1], kv_len)
    for most in (None, max(length, 40)):
        check(ops.paged_attention_fp4(**call, max_kv_len=most), *want, max(kv_len), True)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 8, 15, 16, 17, 24, 31, 32, 33, 40, 64])
def test_group_sizes(gpu_lib, g):
    for hk, q_len in ((1, [1, 1]), (2, [1, 3])):
        kv_len = [333, 70]
        call, k, v = make(BF, g * hk, hk, 64, q_len, kv_len, 16, seed=g)
        check(ops.paged_attention_fp4(**call), *oracle.attention(_np(call["q"]), k, v, q_len, kv_len), 333, True)


def test_split_histories(gpu_lib):
    # Long enough to be cut over workgroups; short ones beside it are done in their first part.
    for dtype, h, hk, d, rows in ((BF, 8, 2, 128, 1), (BF, 4, 4, 64, 1), (BF, 2, 1, 64, 70), (F32, 2, 1, 64, 1)):
        kv_len, q_len = [6000, 1, 900, 0], [rows, 1, rows, 1]
        call, k, v = make(dtype, h, hk, d, q_len, kv_len, 16, seed=rows)
        assert ops.paged_fp4_workspace_size(4, sum(q_len), h, hk, d, 6000, dtype) > 0
        want = oracle.attention(_np(call["q"]), k, v, q_len, kv_len)
        check(ops.paged_attention_fp4(**call, max_kv_len=6000), *want, 6000, dtype == BF)


def test_scales_of_any_size(gpu_lib):
    # Blocks whose scales lie far apart, down to the smallest and up to 2^60.
    for dtype in (BF, F32):
        call, _, _ = make(dtype, 4, 2, 64, [1, 3], [100, 60], 16, seed=5)
        raw = call["pages"].cpu().numpy()
        rng = np.random.default_rng(5)
        n = 2 * 64
        raw[..., n:n + 4] = rng.integers(100, 130, raw[..., n:n + 4].shape)          # K
        raw[..., n + 4:n + 8] = rng.integers(1, 188, raw[..., n + 4:n + 8].shape)     # V
        call["pages"] = torch.from_numpy(raw).cuda()
        k, v = [], []
        for s, length in zip(call["slots"].tolist(), (100, 60)):
            ids = call["page_table"].cpu().numpy()[s, :-(-length // 16)]
            kv = layer.unpack(raw[ids].reshape(-1, raw.shape[2])[:length], 2, 64)
            k.append(kv[:, 0])
            v.append(kv[:, 1])
        want = oracle.attention(_np(call["q"]), np.concatenate(k), np.concatenate(v), [1, 3], [100, 60])
        check(ops.paged_attention_fp4(**call), *want, 100, dtype == BF)


def held(call, hk, d, kv_len):
    """K and V of the packed histories as the call's pages hold them."""
    raw, page = call["pages"].cpu().numpy(), call["pages"].shape[1]
    table = call["page_table"].cpu().numpy()
    rows = [raw[table[s, :-(-n // page)]].reshape(-1, raw.shape[2])[:n] for s, n in zip(call["slots"].tolist(), kv_len)]
    kv = layer.unpack(np.concatenate(rows), hk, d)
    return kv[:, 0], kv[:, 1]


KERNELS = [  # dtype, H, H_kv, d, query rows, history rows: few rows, tiles, and the general kernel
    (BF, 4, 2, 128, [1, 3], [300, 60]), (BF, 8, 1, 64, [1, 1], [1500, 33]), (BF, 2, 1, 96, [1, 9], [99, 40]),
    (BF, 2, 1, 128, [40, 90], [700, 90]), (BF, 2, 2, 64, [130, 65], [200, 65]), (BF, 2, 1, 96, [50, 40], [333, 40]),
    (BF, 2, 1, 256, [1, 30], [70, 200]), (F32, 4, 2, 64, [1, 30], [400, 90]), (F32, 1, 1, 224, [4], [70])]
kernels = pytest.mark.parametrize("dtype, h, hk, d, q_len, kv_len", KERNELS,
                                  ids=lambda v: str(v)[6:] if isinstance(v, torch.dtype) else str(v))


@kernels
def test_scale_bytes_of_zero(gpu_lib, dtype, h, hk, d, q_len, kv_len):
    # E = 0 is 2^-127: K under queries of 2^124, then V. What is below 2^-126 has steps of 2^-133 in
    # bf16, of which a rounding is off by half.
    call, k, v = make(dtype, h, hk, d, q_len, kv_len, 16, seed=d)
    raw = call["pages"].cpu().numpy()
    at, n = hk * d, hk * d // 32
    low = raw.copy()
    low[..., at:at + n] = 0
    small = {**call, "pages": torch.from_numpy(low).cuda(), "q": call["q"] * 2.0 ** 124}
    want = oracle.attention(_np(small["q"]), held(small, hk, d, kv_len)[0], v, q_len, kv_len, scale=1.0)
    check(ops.paged_attention_fp4(**small, scale=1.0), *want, max(kv_len), dtype == BF)
    low = raw.copy()
    low[..., at + n:at + 2 * n] = 0
    small = {**call, "pages": torch.from_numpy(low).cuda()}
    got = _np(ops.paged_attention_fp4(**small)) * 2.0 ** 127
    want, mean, err = oracle.attention(_np(call["q"]), k, held(small, hk, d, kv_len)[1] * 2.0 ** 127, q_len, kv_len)
    step = 2.0 ** -8 if dtype == BF else 0.0
    longest = max(kv_len)
    tol = mean * (2 * err[..., None] + 2 * step + (2 * longest + 64) * oracle.U32) + longest * 2.0 ** -22
    tol = tol + (step if dtype == BF else oracle.U32) * (np.abs(want) + tol) + (2.0 ** -7 if dtype == BF else 0.0)
    off = np.abs(got - want)
    assert np.all(off <= tol), (off.max(), np.abs(want).max(), np.abs(got).max())


def test_every_scale_byte_reads_back(gpu_lib):
    # All codes under all scales, 255 among them: a value is what the form says, exactly.
    hk, d = 2, 128
    rows = np.zeros((256, layer.row_bytes(hk, d)), np.uint8)
    pair = np.arange(hk * d, dtype=np.uint8)
    rows[:, :hk * d] = (pair % 16) | ((pair // 16) << 4)
    rows[:, hk * d:hk * d + hk * d // 16] = np.arange(256)[:, None]
    pool = torch.from_numpy(rows.reshape(16, 16, -1)).cuda()
    at = dev_i32(np.arange(256))
    want = layer.unpack(rows, hk, d)
    exact = np.abs(want) < 2.0 ** 128                      # past that the types have no value
    for dtype in (BF, F32):
        got = _np(ops.cache_read_fp4(at, pool, hk, d, dtype=dtype))
        assert np.array_equal(got[exact], want[exact]) and np.all(np.isnan(got[255]))
        assert np.array_equal(np.signbit(got[exact]), np.signbit(want[exact]))


@kernels
def test_nan_and_infinite_queries_stay_by_themselves(gpu_lib, dtype, h, hk, d, q_len, kv_len):
    # One head of a row NaN; one at minus infinity in a dim where its keys are positive (no key has
    # weight: zeros).
    call, _, v = make(dtype, h, hk, d, q_len, kv_len, 16, seed=d + 1)
    raw = call["pages"].cpu().numpy()
    dim = d - 3
    raw[..., dim // 2] = (raw[..., dim // 2] & 0x0f) | 0x20 if dim % 2 else (raw[..., dim // 2] & 0xf0) | 0x02
    call["pages"] = torch.from_numpy(raw).cuda()
    k = held(call, hk, d, kv_len)[0]
    want, mean, err = oracle.attention(_np(call["q"]), k, v, q_len, kv_len)
    for value, there in ((float("nan"), np.isnan), (-float("inf"), lambda x: x == 0)):
        q = call["q"].clone()
        row = sum(q_len) - 1
        q[row, 0, dim] = value                              # head 0 reads K/V head 0
        got = ops.paged_attention_fp4(**{**call, "q": q})
        assert np.all(there(_np(got)[row, 0]))
        got[row, 0] = torch.from_numpy(want[row, 0]).to(got)
        check(got, want, mean, err, max(kv_len), dtype == BF)


@pytest.mark.parametrize("h, hk, d, q_len, kv_len", [
    (8, 8, 64, [1] * 24, [6000, 3] + [50] * 22), (8, 4, 128, [1, 2, 1], [6000, 1, 900]),
    (2, 1, 64, [70, 33], [5000, 90]), (2, 2, 96, [1, 3], [5000, 70])])
def test_unaligned_queries_over_split_histories(gpu_lib, h, hk, d, q_len, kv_len):
    # bf16 queries off 16 bytes, or off 16 bytes a row: the general kernel under the other kernels' plans.
    call, k, v = make(BF, h, hk, d, q_len, kv_len, 16, seed=h + d)
    n = sum(q_len)
    assert ops.paged_fp4_workspace_size(len(q_len), n, h, hk, d, max(kv_len), BF) > 0
    for lo, pad in ((1, 7), (4, 0), (0, 5)):
        wide = torch.randn(n, h * d + lo + pad, device="cuda").to(BF)
        q = wide[:, lo:lo + h * d].unflatten(1, (h, d))
        got = ops.paged_attention_fp4(**{**call, "q": q}, max_kv_len=max(kv_len))
        check(got, *oracle.attention(_np(q), k, v, q_len, kv_len), max(kv_len), True)


@pytest.mark.parametrize("dtype, h, hk, d, rows", [(BF, 4, 2, 128, 1), (BF, 8, 1, 64, 3), (BF, 2, 2, 64, 80),
                                                   (BF, 2, 1, 96, 40), (F32, 4, 2, 64, 5)])
def test_nan_blocks_reach_only_the_rows_that_see_them(gpu_lib, dtype, h, hk, d, rows):
    kv_len, q_len = [200, 150], [rows, rows]
    call, k, v = make(dtype, h, hk, d, q_len, kv_len, 16, seed=rows)
    clean = ops.paged_attention_fp4(**call)
    raw = call["pages"].cpu().numpy()
    # A block of V in the last key of request 0, one of K in the first key of request 1's last rows.
    slot = call["slots"].tolist()
    table = call["page_table"].cpu().numpy()
    hit = raw.copy()
    hit[table[slot[0], 199 // 16], 199 % 16, hk * d + hk * d // 32] = 255            # V scale 0 of head 0
    hit[table[slot[1], 149 // 16], 149 % 16, hk * d] = 255                            # K scale 0 of head 0
    got = ops.paged_attention_fp4(**{**call, "pages": torch.from_numpy(hit).cuda()})
    g = h // hk
    odd = torch.zeros_like(got, dtype=torch.bool)
    odd[rows - 1, :g, :32] = True                     # only the last row sees the last key
    odd[2 * rows - 1, :g] = True
    assert torch.equal(torch.isnan(got), odd)
    near = (got.float() - clean.float()).abs()[~odd]
    assert torch.all(near <= 2.0 ** -7 * clean.float().abs()[~odd] + 2.0 ** -6)


def test_rows_behind_the_last_request_stay(gpu_lib):
    for rows, length in ((1, 5000), (1, 40), (60, 300)):
        q_len, kv_len = [rows, rows], [length, 30]
        call, k, v = make(BF, 4, 2, 64, q_len, kv_len, 16)
        want = ops.paged_attention_fp4(**call)
        q = torch.cat([call["q"], torch.randn(5, 4, 64, device="cuda").to(BF)])
        out = torch.full_like(q, 7.0)
        ops.paged_attention_fp4(**{**call, "q": q}, out=out)
        assert torch.all(out[2 * rows:] == 7.0)
        check(out[:2 * rows], *oracle.attention(_np(call["q"]), k, v, q_len, kv_len), length, True)
        assert want.shape == call["q"].shape


def test_strided_queries_and_bad_device_data(gpu_lib):
    call, k, v = make(BF, 4, 2, 64, [1, 2], [90, 40], 16)
    wide = torch.randn(3, 8 * 64, device="cuda").to(BF)
    for lo in (0, 8, 3):
        q = wide[:, lo:lo + 256].unflatten(1, (4, 64))
        got = ops.paged_attention_fp4(**{**call, "q": q})
        check(got, *oracle.attention(_np(q), k, v, [1, 2], [90, 40]), 90, True)
    # Page ids, slots and lengths out of range are clamped: finite or NaN, never a fault.
    bad = {**call, "page_table": torch.full_like(call["page_table"], 1 << 30),
           "kv_lens": torch.full_like(call["kv_lens"], 1 << 30), "slots": dev_i32([-1, 99])}
    assert ops.paged_attention_fp4(**bad).shape == (3, 4, 64)
    none = {**call, "kv_lens": torch.full_like(call["kv_lens"], -5)}
    assert torch.all(ops.paged_attention_fp4(**none) == 0)


def test_captured_and_on_another_stream(gpu_lib):
    for q_len, kv_len in (([1, 1, 1], [5000, 3, 700]), ([70, 1], [300, 90])):
        call, _, _ = make(BF, 4, 2, 128, q_len, kv_len, 16)
        kw = dict(max_kv_len=max(kv_len))
        want = ops.paged_attention_fp4(**call, **kw)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        on_side = ops.paged_attention_fp4(**call, **kw, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(on_side, want)
        out = torch.empty_like(want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ops.paged_attention_fp4(**call, **kw, out=out)
        for i in range(3):
            call["q"].copy_(torch.randn_like(call["q"]))
            out.zero_()
            g.replay()
            want = ops.paged_attention_fp4(**call, **kw)
            torch.cuda.synchronize()
            assert torch.equal(out, want)
