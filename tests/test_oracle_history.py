"""Pins of the history oracle: attention against loops, closed forms and torch's own attention,
the cache against the rows that went into it."""

import numpy as np
import pytest
import torch

from oracle import history as oracle


def _case(h, hk, d, q_len, kv_len, seed=0):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((sum(q_len), h, d)), rng.standard_normal((sum(kv_len), hk, d)),
            rng.standard_normal((sum(kv_len), hk, d)))


def test_attention_by_loops():
    q_len, kv_len = [3, 1, 2], [3, 6, 1]
    q, k, v = _case(4, 2, 5, q_len, kv_len)
    rng = np.random.default_rng(1)
    kw = dict(prefix=[0, 2, 9], q_docs=rng.integers(0, 2, 6), kv_docs=rng.integers(0, 2, 10),
              slopes=np.array([0.5, 0.25, 0.1, 0.0]), cap=1.5, scale=0.7)
    got = oracle.attention(q, k, v, q_len, kv_len, **kw)[0]
    a = b = 0
    for r in range(3):
        for i in range(q_len[r]):
            p = kv_len[r] - q_len[r] + i
            for h in range(4):
                s, vs = [], []
                for j in range(kv_len[r]):
                    if (j <= p or j < kw["prefix"][r]) and kw["q_docs"][a + i] == kw["kv_docs"][b + j]:
                        x = sum(q[a + i, h, e] * k[b + j, h // 2, e] for e in range(5)) * 0.7
                        s.append(1.5 * np.tanh(x / 1.5) - kw["slopes"][h] * abs(p - j))
                        vs.append(v[b + j, h // 2])
                want = np.zeros(5)
                if s:
                    w = np.exp(np.array(s))
                    want = sum(x * y for x, y in zip(w / w.sum(), vs))
                assert np.allclose(got[a + i, h], want, rtol=1e-12, atol=1e-12)
        a += q_len[r]
        b += kv_len[r]


@pytest.mark.parametrize("causal", [True, False])
def test_attention_is_torchs(causal):
    q, k, v = _case(2, 2, 8, [7], [7])
    got = oracle.attention(q, k, v, [7], [7], causal=causal)[0]
    t = [torch.from_numpy(x).transpose(0, 1) for x in (q, k, v)]
    want = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=causal)
    assert np.allclose(got, want.transpose(0, 1).numpy(), rtol=1e-12)


def test_attention_closed_forms():
    q, k, v = _case(1, 1, 4, [3], [3])
    got = oracle.attention(q, k * 0, v, [3], [3])[0]          # equal scores: running means
    assert np.allclose(got[:, 0], np.cumsum(v[:, 0], 0) / np.arange(1, 4)[:, None])
    got = oracle.attention(q, k, v, [3], [3], slopes=np.array([1e3]))[0]     # only the row itself
    assert np.allclose(got, v)
    small = oracle.attention(q * 1e-3, k, v, [3], [3], cap=50.0)[0]          # a cap far away
    assert np.allclose(small, oracle.attention(q * 1e-3, k, v, [3], [3])[0], atol=1e-9)
    assert np.all(oracle.attention(q, k[:0], v[:0], [3], [0])[0] == 0)


def test_cache_keeps_every_history():
    rng = np.random.default_rng(0)
    c, want, at = oracle.Cache(2, 60, 3, 8, 10), {s: [] for s in range(8)}, 0
    for _ in range(200):
        kind = rng.integers(4)
        if kind < 2:
            slots, counts = rng.choice(8, 3, replace=False), rng.integers(0, 6, 3)
            rows, code = c.reserve(list(slots), list(counts))
            if code == (0, 0):
                ids = list(range(at, at + counts.sum()))
                at += counts.sum()
                for layer in range(2):
                    c.write(layer, rows, ids)
                for s, n in zip(slots, counts):
                    want[s] += ids[:n]
                    ids = ids[n:]
        elif kind == 2:
            a, b = rng.choice(8, 2, replace=False)
            if c.fork([a], [b]) == (0, 0):
                want[b] = list(want[a])
        else:
            s = rng.integers(8)
            c.free([s, s])
            want[s] = []
            if rng.integers(2):
                n = c.compact()[1]
                assert all(x > 0 for x in c.refs[:n]) and not any(c.refs[n:])
        for s in range(8):
            assert c.history(0, s) == c.history(1, s) == want[s]
        held = [p for row in c.table for p in row if p >= 0]
        assert all(c.refs[p] == held.count(p) for p in range(60))
