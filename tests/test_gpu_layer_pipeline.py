"""GPU: adapters, rotated appends and attention over 4 bits together, as a serving loop uses them:
batches of new events are projected with their requests' adapters, appended to a cache in 4 bits and
encoded over it, and candidates attend over the pages, while slots are forked, freed and compacted in
between. Attention is compared with the oracle over the values that the cache holds, and those with
the rows that went in."""

import numpy as np
import pytest
import torch

from gpu_util import assert_close, dev_bf16, dev_i32, host
from oracle import history as oracle
from oracle import ikbo, layer
from oracle.bf16 import round_bf16
from paper_2607_27744_amd import ops, pipelines
from paper_2607_27744_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _held(p, slot):
    """Every row that a slot holds, as values [L, 2, kv_heads, d]."""
    n = int(p.lens[slot])
    if n == 0:
        return np.zeros((0, 2, p.hk, p.d))
    j = torch.arange(n, device="cuda")
    rows = p.table[slot][(j // p.page)] * p.page + j % p.page
    return host(ops.cache_read_fp4(rows.int(), p.pool[0], p.hk, p.d))


@pytest.mark.parametrize("head_dim, kv_heads, page", [(64, 2, 16), (128, 4, 64), (32, 1, 24), (96, 2, 7)])
def test_ranking_with_adapters_over_four_bits(gpu_lib, head_dim, kv_heads, page):
    counts = [33, 1, 0, 140, 7]
    events = [[70, 1, 40, 129, 0], [1, 1, 1, 1, 1], [9, 0, 3, 64, 2], [1, 1, 1, 1, 1]]
    w = wl.history_case(counts, events, heads=4, kv_heads=kv_heads, head_dim=head_dim, seed=3)
    ad = wl.adapters_of(w, 3, 8, seed=4)
    p = pipelines.prepare_adapted_cache(w, ad, pages=140, page_size=page, table_width=50, slots=8,
                                        base=100.0)
    freqs = host(p.freqs)
    wqkv = np.concatenate([w.wq_s, w.wkv])
    rows_in = {s: np.zeros((0, 2, kv_heads, head_dim)) for s in range(8)}
    slot_of, ids = np.array([6, 0, 3, 5, 1]), np.array([2, -1, 0, 1, 7])
    h, d = 4, head_dim
    for i, b in enumerate(w.batches):
        slots, new = dev_i32(slot_of), np.diff(b.offsets)
        got = pipelines.adapted_step(p, slots, dev_i32(ids), dev_bf16(b.s), dev_i32(b.offsets),
                                     dev_bf16(b.e_c), dev_i32(b.cand_offsets),
                                     max_kv_len=None if i % 2 else 400)
        ops.cache_check(got["status"])
        qkv = round_bf16(layer.adapter_linear(b.s, wqkv, ad.a, ad.b, new, ids, ad.scales)[0])
        qkv = qkv.reshape(-1, h + 2 * kv_heads, d)
        lens = np.zeros(8, int)
        lens[slot_of] = [rows_in[s].shape[0] + n for s, n in zip(slot_of, new)]
        pos = layer.positions(new, slot_of, lens)
        k = layer.rotate(qkv[:, h:h + kv_heads], pos, freqs)
        put = np.stack([k, qkv[:, h + kv_heads:]], 1)
        for r, s in enumerate(slot_of):
            rows_in[s] = np.concatenate([rows_in[s], put[b.offsets[r]:b.offsets[r + 1]]])
        held = [_held(p, s) for s in slot_of]
        for kv, s in zip(held, slot_of):
            # A value is off by at most the scale of its block (1/3.5 of the largest) and what the
            # projection's own rounding moves; in the mean by far less.
            assert kv.shape == rows_in[s].shape
            if kv.size:
                assert np.linalg.norm(kv - rows_in[s]) <= 0.15 * np.linalg.norm(rows_in[s])
        kv = np.concatenate(held)
        n_kv = [x.shape[0] for x in held]
        q = round_bf16(layer.rotate(qkv[:, :h], pos, freqs))
        want = oracle.attention(q, kv[:, 0], kv[:, 1], new, n_kv)[0]
        assert_close(host(got["events"]), round_bf16(want), f"batch {i} events", atol=3e-2)
        q_c = round_bf16(ikbo.linear(b.e_c, w.wq_c)).reshape(-1, h, d)
        q_c = round_bf16(layer.rotate(q_c, np.repeat(lens[slot_of], counts), freqs))
        want = oracle.attention(q_c, kv[:, 0], kv[:, 1], counts, n_kv, causal=False)[0]
        assert_close(host(got["candidates"]), round_bf16(want), f"batch {i} candidates", atol=3e-2)
        if i == 1:
            # Slot 3 is handed to 7 (full pages shared), given back, and the cache compacted.
            before = _held(p, 3)
            st = ops.cache_fork(dev_i32([3]), dev_i32([7]), p.table, p.lens, p.refs, p.pool)
            ops.cache_check(st)
            ops.cache_free(dev_i32([3, 0]), p.table, p.lens, p.refs, p.page)
            ops.cache_check(ops.cache_compact(p.table, p.lens, p.refs, p.pool))
            assert np.array_equal(_held(p, 7), before)
            rows_in[7], rows_in[3], rows_in[0] = rows_in[3], rows_in[3][:0], rows_in[0][:0]
            slot_of[2] = 7


def test_pages_copied_between_pools(gpu_lib):
    # Rows appended to one cache are read and attended to from another that its pages are copied to.
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g).cuda().bfloat16()   # noqa: E731
    src, table, lens, refs = ops.cache_pool_fp4(2, 9, 16, 2, 64, slots=1, table_width=6)
    off = dev_i32([0, 70])
    rows, status = ops.cache_reserve(dev_i32([0]), off, 70, table, lens, refs, 16)
    ops.cache_check(status)
    for one in range(2):
        ops.cache_append(rnd(70, 2, 64), rnd(70, 2, 64), rows, src[one])
    dst = torch.full((2, 12, *src.shape[2:]), 255, dtype=torch.uint8, device="cuda")
    to = dev_i32([11, 0, 7, 3, 5])
    ops.cache_copy(table[0, :5].contiguous(), to, src, dst)
    there = torch.full_like(table, -1)
    there[0, :5] = to
    j = torch.arange(70, device="cuda")
    moved = (to[j // 16] * 16 + j % 16).int()
    q = rnd(3, 4, 64)
    for one in range(2):
        assert torch.equal(ops.cache_read_fp4(rows, src[one], 2, 64), ops.cache_read_fp4(moved, dst[one], 2, 64))
        call = lambda pool, t: ops.paged_attention_fp4(q, pool, t, lens, dev_i32([0, 3]), kv_heads=2)   # noqa: E731
        assert torch.equal(call(src[one], table), call(dst[one], there))
    rest = [p for p in range(12) if p not in to.tolist()]
    assert torch.all(dst[:, rest] == 255)


def test_a_step_that_finds_no_pages_leaves_the_cache(gpu_lib):
    w = wl.history_case([2, 2], [[20, 30], [40, 60]], kv_heads=1, head_dim=64)
    p = pipelines.prepare_adapted_cache(w, wl.adapters_of(w, 2, 8), pages=4, page_size=16, table_width=8)
    slots, ids = dev_i32([1, 0]), dev_i32([0, 1])
    first, second = w.batches
    call = lambda b: pipelines.adapted_step(p, slots, ids, dev_bf16(b.s), dev_i32(b.offsets),  # noqa: E731
                                            dev_bf16(b.e_c), dev_i32(b.cand_offsets))
    ops.cache_check(call(first)["status"])
    kept = [x.clone() for x in (p.pool, p.table, p.lens, p.refs)]
    with pytest.raises(ops.RocsError, match="pages are missing"):
        ops.cache_check(call(second)["status"])
    assert all(torch.equal(x, y) for x, y in zip(kept, (p.pool, p.table, p.lens, p.refs)))


@pytest.mark.parametrize("bad", [2, 99, -1, -3])
def test_a_step_with_a_slot_out_of_range(gpu_lib, bad):
    # The status says so, the cache is unchanged, and what torch looks up stays within it.
    w = wl.history_case([2, 2], [[20, 30], [40, 60]], kv_heads=1, head_dim=64)
    p = pipelines.prepare_adapted_cache(w, wl.adapters_of(w, 2, 8), pages=20, page_size=16, table_width=8)
    first, second = w.batches
    call = lambda b, slots: pipelines.adapted_step(  # noqa: E731
        p, dev_i32(slots), dev_i32([0, 1]), dev_bf16(b.s), dev_i32(b.offsets), dev_bf16(b.e_c),
        dev_i32(b.cand_offsets))
    ops.cache_check(call(first, [1, 0])["status"])
    kept = [x.clone() for x in (p.pool, p.table, p.lens, p.refs)]
    with pytest.raises(ops.RocsError, match="out of range"):
        ops.cache_check(call(second, [1, bad])["status"])
    assert all(torch.equal(x, y) for x, y in zip(kept, (p.pool, p.table, p.lens, p.refs)))


def test_a_step_in_a_graph(gpu_lib):
    # The whole step captured, replayed for the next batch's events beside eager work.
    w = wl.history_case([5, 3], [[70, 40], [1, 1], [1, 1], [1, 1]], kv_heads=2, head_dim=64)
    ad = wl.adapters_of(w, 2, 8)
    make = lambda: pipelines.prepare_adapted_cache(w, ad, pages=20, page_size=16, table_width=12)  # noqa: E731
    p, eager = make(), make()
    slots, ids = dev_i32([1, 0]), dev_i32([0, 1])
    up = lambda b: (dev_bf16(b.s), dev_i32(b.offsets), dev_bf16(b.e_c), dev_i32(b.cand_offsets))  # noqa: E731
    first = up(w.batches[0])
    for c in (p, eager):
        pipelines.adapted_step(c, slots, ids, *first, max_kv_len=192)
    state = [x.clone() for x in (p.pool, p.table, p.lens, p.refs)]
    x = up(w.batches[1])
    pipelines.adapted_step(p, slots, ids, *x, max_kv_len=192)            # loads what it needs
    for old, cur in zip(state, (p.pool, p.table, p.lens, p.refs)):
        cur.copy_(old)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = pipelines.adapted_step(p, slots, ids, *x, max_kv_len=192)
    for b in w.batches[1:]:
        new = up(b)
        x[0].copy_(new[0])
        x[2].copy_(new[2])
        g.replay()
        want = pipelines.adapted_step(eager, slots, ids, *new, max_kv_len=192)
        torch.cuda.synchronize()
        assert torch.equal(got["events"], want["events"])
        assert torch.equal(got["candidates"], want["candidates"])
        assert torch.equal(p.pool, eager.pool) and torch.equal(p.lens, eager.lens)


@pytest.mark.parametrize("name", ["adapter_linear", "paged_step_fp4", "adapted_step"])
def test_the_variants_run(gpu_lib, name):
    from paper_2607_27744_amd import variants
    line = variants.run(name, steps=2, warmup=1)
    assert line["variant"] == name and line["ms"] > 0 and name in variants.NAMES
