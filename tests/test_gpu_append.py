"""GPU: rows appended to a cache with the position rotation, the 4-bit form, and rows read back.

Tolerance of a turned value: cosine and sine are rounded to fp32 (2^-24 each), so are the two products
and their sum: 3 2^-24 (|x| + |y|), and the rounding to the result's type. In 4 bits a value is off by
at most half the step of the codes around it, of a scale that can be either neighbour's where the block's
largest magnitude is within that tolerance of a border."""

import numpy as np
import pytest
import torch

from gpu_util import dev_f32, dev_i32
from oracle import layer as oracle
from paper_2607_27744_amd import ops

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make(counts, lens, h, hk, d, rot, dtype, page=16, seed=0, slots=None, spare=3):
    """Rows whose places follow ops.cache_reserve: lens are the slots' lengths with them."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    m = int(np.sum(counts))
    slots = rng.permutation(len(lens))[:len(counts)] if slots is None else slots
    qkv = torch.randn(m, (h + 2 * hk) * d, generator=g).to(dtype).cuda()
    pages = -(-m // page) + spare
    rows = rng.permutation(pages * page)[:m]
    freqs = (100.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32)
    return dict(m=m, pages=pages, page=page, q=qkv[:, :h * d].unflatten(1, (h, d)),
                k=qkv[:, h * d:(h + hk) * d].unflatten(1, (hk, d)),
                v=qkv[:, (h + hk) * d:].unflatten(1, (hk, d)), rows=rows, freqs=freqs, slots=slots,
                lens=np.asarray(lens), counts=counts,
                pos=oracle.positions(counts, slots, lens) if m else np.zeros(0, np.int64))


def where(c):
    return dict(offsets=dev_i32(np.concatenate([[0], np.cumsum(c["counts"])])), slots=dev_i32(c["slots"]),
                lens=dev_i32(c["lens"]))


def turned_tol(x, freqs, interleaved):
    """3 2^-24 (|x| + |partner|) for turned dims."""
    a, half = np.abs(x), len(freqs)
    y = np.zeros_like(a)
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[..., p] = y[..., q] = 3 * U32 * (a[..., p] + a[..., q])
    return y


def check_turned(got, x, c, interleaved):
    want = oracle.rotate(_np(x), c["pos"], c["freqs"], interleaved)
    tol = turned_tol(_np(x), c["freqs"], interleaved)
    half_step = 2.0 ** -8 if x.dtype == BF else U32
    tol = tol + half_step * (np.abs(want) + tol)
    assert np.all(np.abs(_np(got) - want) <= tol)


CASES = [  # counts, lens, h, hk, d, rot
    ([1] * 6, [5, 1, 900, 70000, 33, 12], 8, 2, 128, 128),
    ([4, 0, 1, 90], [40, 1, 1, 90], 4, 4, 64, 64),
    ([33], [2000000], 2, 1, 32, 16),
    ([2, 5], [2, 500], 3, 3, 96, 48),
    ([1, 2], [7, 9], 1, 1, 256, 256), ([300, 7], [300, 1000], 4, 2, 160, 80),
]
ODD = [([3, 1, 20], [3, 9, 2000], 3, 2, 18, 18), ([5], [6], 1, 1, 7, 6), ([5], [6], 2, 1, 40, 20),
       ([17], [17], 2, 2, 1, 0)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", CASES + ODD, ids=lambda c: f"{sum(c[0])}x{c[2]}.{c[3]}x{c[4]}r{c[5]}")
def test_rows_into_a_pool_of_their_type(gpu_lib, case, dtype, interleaved):
    c = make(*case, dtype, seed=case[4])
    h, hk, d, rot = case[2:]
    pool = torch.full((c["pages"], c["page"], 2, hk, d), 9.0, dtype=dtype, device="cuda")
    freqs = dev_f32(c["freqs"]) if rot else None
    q = ops.cache_append(c["k"], c["v"], dev_i32(c["rows"]), pool, freqs, q=c["q"],
                         interleaved=interleaved, **where(c))
    check_turned(q, c["q"], c, interleaved)
    flat = pool.view(-1, 2, hk, d)
    at = torch.from_numpy(c["rows"]).cuda()
    check_turned(flat[at, 0], c["k"], c, interleaved)
    assert torch.equal(flat[at, 1], c["v"])
    rest = np.setdiff1d(np.arange(flat.shape[0]), c["rows"])
    assert torch.all(flat[torch.from_numpy(rest).cuda()] == 9.0)
    # The same through rotate(), and with the positions given.
    turn = ops.rotate(c["k"], freqs, interleaved=interleaved, **where(c))
    assert torch.equal(turn, flat[at, 0])
    pos = dev_i32(c["pos"])
    assert torch.equal(ops.rotate(c["q"], freqs, positions=pos, interleaved=interleaved), q)
    again = torch.zeros_like(pool)
    none = ops.cache_append(c["k"], c["v"], dev_i32(c["rows"]), again, freqs, positions=pos,
                            interleaved=interleaved)
    assert none is None and torch.equal(again.view_as(flat)[at], flat[at])


def check_fp4(got, x, tol):
    """got: values out of a 4-bit pool; x what should be there, to `tol`."""
    m, _, hk, d = x.shape
    b, t = x.reshape(-1, 32), tol.reshape(-1, 32)
    g = got.reshape(-1, 32)
    most, slack = np.abs(b).max(1), t.max(1)
    low = oracle.quantise((b * (np.maximum(most - slack, 0) / np.maximum(most, 1e-300))[:, None]))[1]
    high = oracle.quantise(b * ((most + slack) / np.maximum(most, 1e-300))[:, None])[1]
    ok = np.zeros(b.shape, bool)
    for byte in (low, high):
        step = 2.0 ** (byte.astype(np.float64) - 127)
        y = np.abs(b) / step
        half = np.where(y <= 2, 0.25, np.where(y <= 4, 0.5, 1.0)) * step
        ok |= np.abs(g - b) <= half + t
    assert np.all(ok), np.flatnonzero(~ok)[:8]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{sum(c[0])}x{c[2]}.{c[3]}x{c[4]}r{c[5]}")
def test_rows_into_four_bits(gpu_lib, case, dtype, interleaved):
    c = make(*case, dtype, seed=case[4] + 1)
    h, hk, d, _ = case[2:]
    pool = torch.full((c["pages"], c["page"], ops.fp4_row_bytes(hk, d)), 0xa5, dtype=torch.uint8,
                      device="cuda")
    rows = dev_i32(c["rows"])
    q = ops.cache_append(c["k"], c["v"], rows, pool, dev_f32(c["freqs"]), q=c["q"],
                         interleaved=interleaved, **where(c))
    check_turned(q, c["q"], c, interleaved)
    bytes_ = pool.view(-1, pool.shape[2]).cpu().numpy()
    used = hk * d + hk * d // 16
    assert np.all(bytes_[:, used:] == 0xa5)                          # padding is not written
    rest = np.setdiff1d(np.arange(bytes_.shape[0]), c["rows"])
    assert np.all(bytes_[rest] == 0xa5)
    kv = np.stack([oracle.rotate(_np(c["k"]), c["pos"], c["freqs"], interleaved), _np(c["v"])], 1)
    tol = np.stack([turned_tol(_np(c["k"]), c["freqs"], interleaved), np.zeros_like(_np(c["v"]))], 1)
    got = oracle.unpack(bytes_[c["rows"]], hk, d)
    check_fp4(got, kv, tol)
    assert np.array_equal(oracle.unpack(oracle.pack(kv), hk, d)[:, 1], got[:, 1])     # V is exact
    for out in (BF, F32):
        back = ops.cache_read_fp4(rows, pool, hk, d, dtype=out)
        assert back.dtype == out and np.array_equal(_np(back), got)


def test_codes_at_every_border(gpu_lib):
    # Ties, scale borders, zeros, the largest and smallest magnitudes: the oracle's bytes.
    edge = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 6.5, 7], np.float32)
    x = np.zeros((40, 64), np.float32)
    for i in range(40):
        top = [4, 6, 7, 7.001, 7.5, 8, 3.4, 3.5, 3.51, 0][i % 10]
        x[i, :17] = edge * (np.float32(top) / 8 if i % 3 else 1)
        x[i, 17:34] = -x[i, :17]
        x[i, 34] = top
        x[i] *= np.float32(2.0) ** [0, -3, 40, -140, 120, -126, 1, -127, 124, -100][i // 4]
    x[39, :3] = [3.4e38, -3.4e38, 1e-45]
    assert np.all(np.isfinite(x))
    x = x.reshape(40, 1, 64)
    pool = torch.zeros((3, 16, 80), dtype=torch.uint8, device="cuda")
    rows = dev_i32(np.arange(40))
    ops.cache_append(dev_f32(x), dev_f32(-x), rows, pool)
    want = oracle.unpack(oracle.pack(np.stack([x, -x], 1).astype(np.float64)), 1, 64)
    got = oracle.unpack(pool.view(-1, 80).cpu().numpy()[:40], 1, 64)
    assert np.array_equal(got, want)
    flat = pool.view(-1, 80)[:40].cpu().numpy()
    assert np.array_equal(flat[:, 64:68], oracle.pack(np.stack([x, -x], 1).astype(np.float64))[:, 64:68])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_an_odd_value_makes_its_block_nan(gpu_lib, bad):
    k = torch.randn(5, 2, 64, device="cuda").to(BF)
    v = k.clone()
    k[1, 0, 3], v[4, 1, 63] = bad, bad
    pool = torch.zeros((1, 8, ops.fp4_row_bytes(2, 64)), dtype=torch.uint8, device="cuda")
    rows = dev_i32(np.arange(5))
    ops.cache_append(k, v, rows, pool)
    got = ops.cache_read_fp4(rows, pool, 2, 64)
    odd = torch.zeros_like(got, dtype=torch.bool)
    odd[1, 0, 0, :32] = odd[4, 1, 1, 32:] = True
    assert torch.equal(torch.isnan(got), odd)


@pytest.mark.parametrize("fp4", [False, True])
def test_rows_outside_and_a_padded_batch(gpu_lib, fp4):
    c = make([3, 2], [10, 20], 2, 1, 64, 64, BF, seed=3)
    pad = 4
    big = make([3, 2, pad], [10, 20, 9], 2, 1, 64, 64, BF, seed=3)
    rows = np.concatenate([c["rows"], np.arange(40, 40 + pad)])
    rows[1], rows[4] = -1, 1 << 30
    shape = (4, 16, 80) if fp4 else (4, 16, 2, 1, 64)
    pool = torch.full(shape, 3, dtype=torch.uint8 if fp4 else BF, device="cuda")
    out = torch.full((5 + pad, 2, 64), 7.0, dtype=BF, device="cuda")
    w = where(c)
    ops.cache_append(big["k"], big["v"], dev_i32(rows), pool, dev_f32(c["freqs"]), q=big["q"], q_out=out, **w)
    assert torch.all(out[5:] == 7.0)                                 # rows behind the last request
    pos = dev_i32(np.concatenate([oracle.positions([3, 2], c["slots"], c["lens"]), np.zeros(pad, int)]))
    assert torch.equal(out[:5], ops.rotate(big["q"], dev_f32(c["freqs"]), positions=pos)[:5])
    flat = pool.view(64, -1)
    written = sorted(rows[i] for i in (0, 2, 3))
    rest = np.setdiff1d(np.arange(64), written)
    assert torch.all(flat[torch.from_numpy(rest).cuda()] == 3)
    assert not torch.any(torch.all(flat[torch.tensor(written).cuda()] == 3, 1))
    if fp4:
        back = ops.cache_read_fp4(dev_i32(rows), pool, 1, 64)
        assert torch.all(back[[1, 4]] == 0) and not torch.any(torch.all(back[[0, 2, 3]].flatten(1) == 0, 1))


@pytest.mark.parametrize("r", [1, 63, 64, 65, 500, 5000])
def test_requests_are_found(gpu_lib, r):
    # Ragged requests, empty ones among them: every row gets its own position.
    rng = np.random.default_rng(r)
    counts = rng.integers(0, 4, r)
    counts[rng.integers(r)] = 5
    lens = counts + rng.integers(0, 1000, r)
    c = make(counts, lens, 1, 1, 2, 2, F32, seed=r, slots=rng.permutation(r))
    lens_by_slot = np.empty(r, int)
    lens_by_slot[c["slots"]] = lens
    c["lens"], c["pos"] = lens_by_slot, oracle.positions(counts, c["slots"], lens_by_slot)
    check_turned(ops.rotate(c["q"], dev_f32(c["freqs"]), **where(c)), c["q"], c, False)


def test_far_and_negative_positions(gpu_lib):
    pos = np.array([0, 1, -1, 65537, 1 << 20, (1 << 30) + 1, (1 << 31) - 1, -(1 << 31)])
    x = torch.randn(8, 3, 64, device="cuda")
    c = dict(pos=pos, freqs=(np.float32(10000.0) ** (-np.arange(32) / 32)).astype(np.float32))
    got = ops.rotate(x, dev_f32(c["freqs"]), positions=dev_i32(pos))
    want = oracle.rotate(_np(x), pos, c["freqs"])
    # p f and its reduction in 64 bits: 2^31 turns leave 2^-22 of a radian.
    far = np.abs(pos)[:, None, None] * 2.0 ** -50
    tol = turned_tol(_np(x), c["freqs"], False) * (1 + far / U32) + U32 * np.abs(want)
    assert np.all(np.abs(_np(got) - want) <= tol)


def test_captured_and_on_another_stream(gpu_lib):
    c = make([1, 30, 2], [50, 30, 8], 4, 2, 64, 64, BF)
    rows, freqs, w = dev_i32(c["rows"]), dev_f32(c["freqs"]), where(c)
    pools = [torch.zeros((c["pages"], 16, ops.fp4_row_bytes(2, 64)), dtype=torch.uint8, device="cuda")
             for _ in range(3)]
    want = ops.cache_append(c["k"], c["v"], rows, pools[0], freqs, q=c["q"], **w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = ops.cache_append(c["k"], c["v"], rows, pools[1], freqs, q=c["q"], stream=side, **w)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(on_side, want) and torch.equal(pools[1], pools[0])
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ops.cache_append(c["k"], c["v"], rows, pools[2], freqs, q=c["q"], q_out=out, **w)
    for i in range(3):
        c["k"].copy_(torch.randn_like(c["k"]))
        out.zero_()
        pools[2].zero_()
        g.replay()
        want = ops.cache_append(c["k"], c["v"], rows, pools[0], freqs, q=c["q"], **w)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(pools[2], pools[0])
