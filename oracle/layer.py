"""Float64 oracle of a projection with low-rank adapters, the position rotation and the cache's
4-bit form, from their definitions (include/rocs_layer.h), row by row where that is plainest.
"""

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def adapter_linear(x, w, a, b, counts, ids, scales=None, bias=None, relu=False):
    """(out, t of the rows, weight of |b| |t|, weight of |x| |w|): t [N, rank] is s A x, zero
    without an adapter."""
    n, rank = x.shape[0], a.shape[1]
    out, t = x @ w.T, np.zeros((n, rank))
    move = np.zeros_like(out)
    at = 0
    for c, i in zip(counts, ids):
        if 0 <= i < a.shape[0]:
            s = 1.0 if scales is None else scales[i]
            t[at:at + c] = s * (x[at:at + c] @ a[i].T)
            out[at:at + c] += t[at:at + c] @ b[i].T
            move[at:at + c] = np.abs(t[at:at + c]) @ np.abs(b[i]).T
        at += c
    if bias is not None:
        out = out + bias
    if relu:
        out = np.maximum(out, 0.0)
    return out, t, move, np.abs(x) @ np.abs(w).T


def positions(counts, slots, lens):
    """Positions of packed rows that are the last of their slots' histories."""
    return np.concatenate([lens[s] - c + np.arange(c) for c, s in zip(counts, slots)]).astype(np.int64)


def rotate(x, pos, freqs, interleaved=False):
    """x [M, heads, d] turned by pos * freqs."""
    y = np.array(x, np.float64)
    half = len(freqs)
    for i, f in enumerate(np.asarray(freqs, np.float64)):
        t = np.asarray(pos, np.float64)[:, None] * f
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        y[..., p] = x[..., p] * np.cos(t) - x[..., q] * np.sin(t)
        y[..., q] = x[..., p] * np.sin(t) + x[..., q] * np.cos(t)
    return y


def row_bytes(kv_heads, d):
    return -(-kv_heads * d * 17 // 256) * 16 if kv_heads * d % 16 == 0 else None


def quantise(x):
    """x [..., d]: (codes [..., d], scale bytes [..., d / 32])."""
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK)
    codes = np.zeros(blocks.shape, np.uint8)
    scale = np.zeros(blocks.shape[:-1], np.uint8)
    for at in np.ndindex(scale.shape):
        v = blocks[at]
        if not np.all(np.isfinite(v)):
            scale[at] = 255
            continue
        m = np.max(np.abs(v))
        e = -126 if m == 0 else int(np.floor(np.log2(m))) - 2
        if m > 0 and m / 2.0 ** e > 7:
            e += 1
        e = min(max(e, -126), 125)
        scale[at] = e + 127
        y = np.abs(v) / 2.0 ** e
        off = np.abs(y[:, None] - GRID[None, :])
        near = off == off.min(1, keepdims=True)                  # two of them at a tie: the even code
        code = np.array([next((c for c in np.flatnonzero(row) if c % 2 == 0 or row.sum() == 1))
                         for row in near])
        codes[at] = code + 8 * np.signbit(v)
    return codes.reshape(x.shape), scale


def values(codes, scale):
    """Codes and scale bytes as values; a block of scale 255 is NaN."""
    v = GRID[codes % 8] * np.where(codes >= 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (v.reshape(*scale.shape, BLOCK) * s[..., None]).reshape(codes.shape)


def pack(kv):
    """kv [M, 2, kv_heads, d] -> rows of bytes."""
    m, _, hk, d = kv.shape
    codes, scale = quantise(kv)
    codes = codes.reshape(m, -1)
    rows = np.zeros((m, row_bytes(hk, d)), np.uint8)
    rows[:, :hk * d] = codes[:, 0::2] | codes[:, 1::2] << 4
    rows[:, hk * d:hk * d + hk * d // 16] = scale.reshape(m, -1)
    return rows


def unpack(rows, hk, d):
    """Rows of bytes -> [M, 2, kv_heads, d]."""
    codes = np.empty((rows.shape[0], 2 * hk * d), np.uint8)
    codes[:, 0::2], codes[:, 1::2] = rows[:, :hk * d] & 15, rows[:, :hk * d] >> 4
    scale = rows[:, hk * d:hk * d + hk * d // 16]
    return values(codes, scale).reshape(-1, 2, hk, d)
